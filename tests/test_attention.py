"""Attention of the training model, its backward pass and the learned position bias, against fp64 with elementwise bounds."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao

DEV = "cuda:0"
T = {"f32": torch.float32, "bf16": torch.bfloat16}
# half a step of the outputs' type; the step the products' operands are rounded with
STEPS = {"f32": (2.0 ** -24, 0.0), "bf16": (2.0 ** -8, 2.0 ** -8)}


@pytest.fixture(scope="module")
def eg():
    from paper_2201_06227_amd import _build, binding
    if _build.is_stale():
        _build.build_library()
    binding.lib()
    return binding


def np64(t):
    return t.detach().double().cpu().numpy()


def make(dtype, b, nq, nk, h, g, d, seed=0, gain=1.0):
    rng = torch.Generator().manual_seed(seed)
    one = lambda *s, k=1.0: (torch.randn(s, generator=rng) * k).to(T[dtype])  # noqa: E731
    return one(b, nq, h, d, k=gain), one(b, nk, g, d, k=gain), one(b, nk, g, d), one(b, nq, h, d)


def close(got, want, bound, what):
    got = np64(got)
    assert got.shape == want.shape, what
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), what
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin]), what
    off = np.abs(got[fin] - want[fin])
    assert (off - bound[fin]).max(initial=-1.0) <= 1e-30, (what, float(off.max()), float((off / np.maximum(bound[fin], 1e-300)).max()))


def run_and_check(eg, dtype, q, k, v, dout, causal=False, q_lens=None, k_lens=None, bias=None, scale=None, grads=None):
    """Forward and backward on the GPU (inputs: CPU tensors or views already there), held to the oracle's bounds."""
    on = lambda t: None if t is None else t.to(DEV) if not t.is_cuda else t  # noqa: E731
    q, k, v, dout = on(q), on(k), on(v), on(dout)
    lens = [None if n is None else torch.tensor(n, dtype=torch.int32, device=DEV) for n in (q_lens, k_lens)]
    pb = None if bias is None else eg.PositionBias(bias[0].to(DEV), bias[1], bias[2])
    how = dict(causal=causal, q_lens=lens[0], k_lens=lens[1], bias=pb, scale=scale)
    out, lse = eg.attention(q, k, v, **how)
    h_out, h_op = STEPS[dtype]
    d = q.shape[3]
    scale = np.float64(np.float32(1.0 / math.sqrt(d) if scale is None else scale))
    ob = None if bias is None else (np64(bias[0]), bias[1], bias[2])
    arr = dict(q=np64(q), k=np64(k), v=np64(v), scale=scale, causal=causal, q_lens=q_lens, k_lens=k_lens, bias=ob, half_step=h_out, operand_step=h_op)
    want = ao.attention(**arr)
    close(out, want["out"], want["bound"]["out"], "out")
    close(lse, want["lse"], want["bound"]["lse"], "lse")
    given = {} if grads is None else dict(zip(("dq", "dk", "dv"), grads))
    dq, dk, dv, dtable = eg.attention_backward(dout, q, k, v, out, lse, **how, **given)
    want = ao.attention(**arr, dout=np64(dout), saved=(np64(out), np64(lse)))
    for name, t in (("dq", dq), ("dk", dk), ("dv", dv)):
        close(t, want[name], want["bound"][name], name)
    if bias is not None:
        close(dtable, want["dtable"], want["bound"]["dtable"], "dtable")
    else:
        assert dtable is None
    return out, lse, dq, dk, dv, dtable


def table(buckets, heads, seed=7, gain=1.0):
    return torch.randn(buckets, heads, generator=torch.Generator().manual_seed(seed)) * gain


# ---- host: definition of the buckets, refusals ----------------------------------------------------------------

def test_oracle_against_differences():
    """The oracle's gradients are those of its forward: central differences in fp64."""
    rng = np.random.default_rng(3)
    b, nq, nk, h, g, d = 2, 5, 7, 4, 2, 3
    x = dict(q=rng.normal(size=(b, nq, h, d)), k=rng.normal(size=(b, nk, g, d)), v=rng.normal(size=(b, nk, g, d)))
    tab, w = rng.normal(size=(6, h)), rng.normal(size=(b, nq, h, d))
    for causal, both in ((False, True), (True, False)):
        how = dict(scale=0.4, causal=causal, q_lens=[5, 3], k_lens=[7, 4])
        f = lambda x, t: (ao.attention(**x, bias=(t, 5, both), **how)["out"] * w).sum()  # noqa: E731
        base = ao.attention(**x, bias=(tab, 5, both), **how)
        grad = ao.attention(**x, bias=(tab, 5, both), **how, dout=w, saved=(base["out"], base["lse"]))
        for name in ("q", "k", "v", "table"):
            step = rng.normal(size=tab.shape if name == "table" else x[name].shape)
            at = lambda e: f(x, tab + e * step) if name == "table" else f({**x, name: x[name] + e * step}, tab)  # noqa: E731
            diff = (at(1e-5) - at(-1e-5)) / 2e-5
            assert abs(diff - (grad["d" + name] * step).sum()) < 1e-7 * (1 + abs(diff)), (causal, name)


@pytest.mark.parametrize("buckets,far,both", [(32, 128, True), (32, 128, False), (8, 16, True), (2, 2, False), (4, 1024, True), (128, 65, False),
                                              (20, 50, True), (14, 1000, True), (127, 1024, False)])
def test_bucket_borders_by_whole_numbers(buckets, far, both):
    """The rule by powers in fp64 that callers are told, at every distance, against whole-number arithmetic."""
    n = buckets // 2 if both else buckets
    e = n // 2
    m = n - e
    for r in range(0, far + 5):
        want = ao.bucket_of(-r, buckets, far, both)
        x = [e * (far / e) ** (k / m) for k in range(m)]
        got = r if r < e else e + max(k for k in range(m) if r >= x[k] - 1e-12 * x[k])
        assert got == want, r
    assert ao.bucket_of(0, buckets, far, both) == 0
    if both:
        assert ao.bucket_of(1, buckets, far, both) == n + 1 if e > 1 else n


def desc(eg, **more):
    d = eg.AttentionDesc(eg.BF16, 2, 4, 2, 16, 24, 32, 0, 0.125, None, None, None)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def heads(eg, n, h, d=32, data=0x1000, **more):
    t = eg.Heads(data, n * h * d, h * d, d)
    for k, v in more.items():
        setattr(t, k, v)
    return t


def test_refusals(eg):
    """Everything that the header calls an error, found on the host: no pointer here is ever read."""
    L, big = eg.lib(), 1 << 30
    fake = ctypes.c_void_p(0x1000)
    tab = eg.PositionTable(0x1000, 32, 128, 1)

    def fwd(d=None, q=None, k=None, v=None, out=None, lse=fake, ws=fake, ws_bytes=big):
        d = desc(eg) if d is None else d
        return L.egeria_attention(d, q or heads(eg, 16, 4), k or heads(eg, 24, 2), v or heads(eg, 24, 2), out or heads(eg, 16, 4), lse, ws, ws_bytes, None)

    def bwd(d=None, lse=fake, dtable=None, ws=fake, ws_bytes=big, **t):
        d = desc(eg) if d is None else d
        shape = dict(dout=(16, 4), q=(16, 4), k=(24, 2), v=(24, 2), out=(16, 4), dq=(16, 4), dk=(24, 2), dv=(24, 2))
        t = {n: t.get(n) or heads(eg, *s) for n, s in shape.items()}
        return L.egeria_attention_backward(d, t["dout"], t["q"], t["k"], t["v"], t["out"], lse, t["dq"], t["dk"], t["dv"], dtable, ws, ws_bytes, None)

    bad = [dict(dtype=2), dict(dtype=-1), dict(batch=-1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(q_len=-1), dict(k_len=-1),
           dict(head_dim=0), dict(scale=math.nan), dict(scale=math.inf), dict(q_lens=0x1002), dict(k_lens=0x1001)]
    for b, far, both in ((32, 128, 1), (3, 128, 1), (5, 128, 1), (1, 128, 0), (130, 512, 0), (32, 8, 1), (32, 16, 0), (32, 1025, 1)):
        if (b, far) != (32, 128):
            t = eg.PositionTable(0x1000, b, far, both)
            bad.append(dict(bias=ctypes.pointer(t)))
    for t in (eg.PositionTable(None, 32, 128, 1), eg.PositionTable(0x1004, 32, 128, 1)):
        bad.append(dict(bias=ctypes.pointer(t)))
    for more in bad:
        assert fwd(desc(eg, **more)) == eg.ERR_INVALID_ARG, more
        assert bwd(desc(eg, **more)) == eg.ERR_INVALID_ARG, more
        assert L.egeria_attention_workspace_bytes(desc(eg, **more), 0) == 0
        assert L.egeria_attention_workspace_bytes(desc(eg, **more), 1) == 0
    assert L.egeria_attention_workspace_bytes(None, 1) == 0
    for more in (dict(head_dim=129), dict(heads=65536, kv_heads=2)):
        assert fwd(desc(eg, **more)) == eg.ERR_UNSUPPORTED and bwd(desc(eg, **more)) == eg.ERR_UNSUPPORTED
    # tensors
    for more in (dict(data=None), dict(data=0x1001), dict(batch_stride=-1), dict(token_stride=-128), dict(head_stride=-32)):
        for n in ("q", "k", "v", "out"):
            assert fwd(**{n: heads(eg, 24 if n in "kv" else 16, 2 if n in "kv" else 4, **more)}) == eg.ERR_INVALID_ARG, (n, more)
        for n in ("dout", "q", "k", "v", "out", "dq", "dk", "dv"):
            key = n in ("k", "v", "dk", "dv")
            assert bwd(**{n: heads(eg, 24 if key else 16, 2 if key else 4, **more)}) == eg.ERR_INVALID_ARG, (n, more)
    # outputs whose elements overlap
    for more in (dict(batch_stride=0), dict(token_stride=0), dict(head_stride=31), dict(token_stride=127), dict(batch_stride=16 * 128 - 1)):
        assert fwd(out=heads(eg, 16, 4, **more)) == eg.ERR_INVALID_ARG, more
        assert bwd(dq=heads(eg, 16, 4, **more)) == eg.ERR_INVALID_ARG, more
    assert bwd(dk=heads(eg, 24, 2, token_stride=32)) == eg.ERR_INVALID_ARG and bwd(dv=heads(eg, 24, 2, head_stride=0)) == eg.ERR_INVALID_ARG
    assert fwd(q=heads(eg, 16, 4, token_stride=1 << 60)) == eg.ERR_UNSUPPORTED
    # the rest
    assert fwd(lse=None) == eg.ERR_INVALID_ARG and fwd(lse=ctypes.c_void_p(0x1004)) == eg.ERR_INVALID_ARG
    assert fwd(ws=None) == eg.ERR_INVALID_ARG and fwd(ws_bytes=8) == eg.ERR_WORKSPACE_TOO_SMALL
    assert bwd(lse=None) == eg.ERR_INVALID_ARG and bwd(ws=None) == eg.ERR_INVALID_ARG and bwd(ws=ctypes.c_void_p(0x1008)) == eg.ERR_INVALID_ARG
    assert bwd(ws_bytes=L.egeria_attention_workspace_bytes(desc(eg), 1) - 1) == eg.ERR_WORKSPACE_TOO_SMALL
    assert bwd(dtable=fake) == eg.ERR_INVALID_ARG                                # no table to take the gradient of
    assert bwd(desc(eg, bias=ctypes.pointer(tab)), dtable=ctypes.c_void_p(0x1004)) == eg.ERR_INVALID_ARG
    assert L.egeria_attention(None, heads(eg, 16, 4), heads(eg, 24, 2), heads(eg, 24, 2), heads(eg, 16, 4), fake, fake, big, None) == eg.ERR_INVALID_ARG
    assert L.egeria_attention(desc(eg), None, heads(eg, 24, 2), heads(eg, 24, 2), heads(eg, 16, 4), fake, fake, big, None) == eg.ERR_INVALID_ARG


def test_position_bias_refusals(eg):
    L, big = eg.lib(), 1 << 30
    fake, odd = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)
    good = eg.PositionTable(0x1000, 32, 128, 1)
    tables = [eg.PositionTable(*x) for x in ((None, 32, 128, 1), (0x1004, 32, 128, 1), (0x1000, 31, 128, 1), (0x1000, 2, 128, 1), (0x1000, 1, 128, 0),
                                             (0x1000, 129, 512, 0), (0x1000, 32, 8, 1), (0x1000, 32, 1025, 1))]
    for t in tables + [None]:
        assert L.egeria_position_bias(t, 4, 8, 8, 0, fake, eg.F32, None) == eg.ERR_INVALID_ARG
        assert L.egeria_position_bias_backward(t, fake, eg.F32, 2, 4, 8, 8, 0, fake, fake, big, None) == eg.ERR_INVALID_ARG
        assert L.egeria_position_bias_workspace_bytes(t, 2, 4, 8, 8, eg.F32) == 0
    for heads_, nq, nk, off, dt in ((0, 8, 8, 0, 0), (65536, 8, 8, 0, 0), (4, -1, 8, 0, 0), (4, 8, -1, 0, 0), (4, 8, 8, (1 << 29) + 1, 0), (4, 8, 8, 0, 5)):
        assert L.egeria_position_bias(good, heads_, nq, nk, off, fake, dt, None) == eg.ERR_INVALID_ARG
        assert L.egeria_position_bias_backward(good, fake, dt, 2, heads_, nq, nk, off, fake, fake, big, None) == eg.ERR_INVALID_ARG
    for p in (None, odd):
        assert L.egeria_position_bias(good, 4, 8, 8, 0, p, eg.F32, None) == eg.ERR_INVALID_ARG
        assert L.egeria_position_bias_backward(good, p, eg.F32, 2, 4, 8, 8, 0, fake, fake, big, None) == eg.ERR_INVALID_ARG
        assert L.egeria_position_bias_backward(good, fake, eg.F32, 2, 4, 8, 8, 0, p, fake, big, None) == eg.ERR_INVALID_ARG
        assert L.egeria_position_bias_backward(good, fake, eg.F32, 2, 4, 8, 8, 0, fake, p, big, None) == eg.ERR_INVALID_ARG
    assert L.egeria_position_bias_backward(good, fake, eg.F32, -1, 4, 8, 8, 0, fake, fake, big, None) == eg.ERR_INVALID_ARG
    need = L.egeria_position_bias_workspace_bytes(good, 2, 4, 8, 8, eg.F32)
    assert need >= 4 * 32 * 4
    assert L.egeria_position_bias_backward(good, fake, eg.F32, 2, 4, 8, 8, 0, fake, fake, need - 1, None) == eg.ERR_WORKSPACE_TOO_SMALL


def test_binding_refuses_other_tensors(eg):
    """Checks of the Python layer, on host tensors (none of which it takes)."""
    q, k = torch.zeros(2, 4, 4, 8), torch.zeros(2, 6, 2, 8)
    with pytest.raises(ValueError):
        eg.attention(q, k, k)                                                    # not on a GPU
    with pytest.raises(ValueError):
        eg.position_bias(eg.PositionBias(torch.zeros(32, 4), 128), 4, 4)
    for bad in ((q[0], k, k), (q, k, k[:, :5]), (q, k[:1], k[:1]), (q, k[..., :4], k[..., :4]), (q, k.bfloat16(), k)):
        with pytest.raises(ValueError):
            eg._attention_desc(*bad, False, None, None, None, None)
    with pytest.raises(ValueError):
        eg._heads(q.transpose(1, 3))                                             # features not contiguous
    for lens in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            eg._lens(lens, 2)
    with pytest.raises(TypeError):
        eg._attention_desc(q.half(), k.half(), k.half(), False, None, None, None, None)


def test_launches_beyond_the_grid(eg):
    """A launch has fewer than 2^32 threads of 256 to a workgroup: more tiles are refused on the host."""
    L, fake, big = eg.lib(), ctypes.c_void_p(0x1000), 1 << 62
    many = desc(eg, batch=1 << 24, heads=1, kv_heads=1, q_len=33, k_len=600, head_dim=1)
    t = lambda n: eg.Heads(0x1000, n, 1, 1)  # noqa: E731
    assert L.egeria_attention(many, t(33), t(600), t(600), t(33), fake, fake, big, None) == eg.ERR_UNSUPPORTED
    one = desc(eg, batch=1 << 24, heads=1, kv_heads=1, q_len=1, k_len=1, head_dim=1)
    assert L.egeria_attention(one, t(1), t(1), t(1), t(1), fake, fake, big, None) == eg.ERR_UNSUPPORTED
    for d, nq, nk in ((many, 33, 600), (one, 1, 1)):
        assert L.egeria_attention_backward(d, t(nq), t(nq), t(nk), t(nk), t(nq), fake, t(nq), t(nk), t(nk), None, fake, big, None) == eg.ERR_UNSUPPORTED
    tab = eg.PositionTable(0x1000, 32, 128, 1)
    assert L.egeria_position_bias(tab, 64, 1 << 28, 1, 0, fake, eg.BF16, None) == eg.ERR_UNSUPPORTED
    assert L.egeria_position_bias_backward(tab, fake, eg.BF16, 1, 64, 1 << 28, 1, 0, fake, fake, big, None) == eg.ERR_UNSUPPORTED


def test_integers_beyond_c(eg):
    """A distance or offset that a C int does not hold is refused, not cut to its low bits."""
    with pytest.raises(ValueError):
        eg._int32(1 << 32)
    with pytest.raises(ValueError):
        eg._int32(-(1 << 31) - 1)
    with pytest.raises(TypeError):
        eg._int32(1.5)
    assert eg._int32(np.int64(7)) == 7 and eg._int32(-(1 << 31)) == -(1 << 31)


# ---- GPU -----------------------------------------------------------------------------------------------------------

SHAPES = [  # batch, q_len, k_len, heads, kv_heads, dim
    (1, 1, 1, 1, 1, 1), (2, 3, 5, 2, 1, 8), (2, 32, 32, 2, 2, 64), (1, 65, 63, 3, 3, 33), (2, 64, 128, 4, 2, 64), (1, 129, 257, 2, 1, 128),
    (3, 31, 200, 6, 2, 40), (1, 200, 31, 4, 4, 80), (1, 1, 300, 8, 2, 128), (2, 7, 513, 8, 2, 64), (1, 197, 197, 3, 3, 64), (1, 130, 130, 1, 1, 127),
    (2, 257, 70, 2, 2, 96), (1, 33, 1025, 4, 1, 16),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("causal", [False, True])
def test_attention_shapes(eg, dtype, shape, causal):
    run_and_check(eg, dtype, *make(dtype, *shape, seed=sum(shape)), causal=causal)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,buckets,far,both,causal", [
    ((2, 70, 70, 4, 2, 64), 32, 128, True, False), ((1, 300, 300, 2, 2, 64), 32, 128, True, False), ((1, 300, 300, 2, 1, 32), 32, 100, False, True),
    ((2, 40, 333, 3, 3, 40), 8, 16, True, False), ((1, 9, 600, 8, 2, 128), 32, 128, False, True), ((2, 1, 400, 4, 4, 64), 20, 50, False, True),
    ((1, 150, 90, 2, 2, 48), 4, 1024, True, True), ((1, 260, 260, 1, 1, 16), 127, 1000, False, False), ((1, 700, 700, 1, 1, 8), 2, 2, False, True),
], ids=str)
def test_attention_position_bias(eg, dtype, shape, buckets, far, both, causal):
    run_and_check(eg, dtype, *make(dtype, *shape, seed=buckets + far), causal=causal, bias=(table(buckets, shape[3]), far, both))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
def test_attention_lengths(eg, dtype, causal, with_bias):
    """Padded batch: full, odd, single-token and empty sequences; more queries than keys; lengths outside the range are clamped."""
    q, k, v, dout = make(dtype, 6, 70, 133, 4, 2, 64, seed=5)
    bias = (table(16, 4), 60, not causal) if with_bias else None
    run_and_check(eg, dtype, q, k, v, dout, causal=causal, bias=bias, q_lens=[70, 33, 0, 1, 70, 99], k_lens=[133, 64, 50, 1, 0, 200])
    run_and_check(eg, dtype, q, k, v, dout, causal=causal, bias=bias, q_lens=[70, 65, 64, 63, 2, -4], k_lens=[3, 65, 17, 128, 1, -1])
    run_and_check(eg, dtype, q, k, v, dout, causal=causal, bias=bias, k_lens=[133, 132, 129, 128, 127, 7])
    run_and_check(eg, dtype, q, k, v, dout, causal=causal, bias=bias, q_lens=[1, 2, 70, 69, 64, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,causal,bias,lens", [
    ((64, 40, 33, 2, 2, 64), False, None, False), ((32, 70, 130, 8, 4, 40), True, None, True), ((43, 130, 200, 3, 3, 64), False, (32, 128, True), True),
    ((130, 5, 256, 1, 1, 33), False, (16, 40, True), False), ((16, 100, 128, 16, 8, 64), True, (32, 128, False), True), ((128, 1, 1, 1, 1, 1), False, None, False),
    ((64, 64, 255, 2, 2, 16), True, (8, 20, True), True), ((32, 300, 64, 4, 4, 48), True, (32, 100, False), True), ((26, 200, 256, 10, 5, 64), False, (20, 50, True), True),
    ((64, 33, 100, 2, 2, 64), False, (4, 1024, True), False), ((65, 100, 130, 8, 4, 32), True, (16, 40, False), True), ((130, 70, 40, 4, 4, 16), False, (16, 40, True), False),
    ((129, 200, 33, 4, 4, 40), True, None, True)], ids=str)
def test_attention_many_short_sequences(eg, dtype, shape, causal, bias, lens):
    """Batches with a workgroup for each key head: few keys, queries of every number, shared key heads, empty sequences."""
    b, nq, nk, h = shape[:4]
    rng = np.random.default_rng(b + nk)
    ql, kl = (rng.integers(0, nq + 1, b), rng.integers(0, nk + 1, b)) if lens else (None, None)
    if lens:
        ql[:4], kl[:4] = [nq, 0, nq, nq], [nk, nk, 0, 1]
    tab = None if bias is None else (table(bias[0], h), bias[1], bias[2])
    run_and_check(eg, dtype, *make(dtype, *shape, seed=b), causal=causal, bias=tab, q_lens=None if ql is None else ql.tolist(), k_lens=None if kl is None else kl.tolist())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nq,nk", [(0, 9), (9, 0), (0, 0)])
def test_attention_many_empty_sequences(eg, dtype, nq, nk):
    q, k, v, dout = make(dtype, 130, nq, nk, 4, 2, 16, seed=1)
    run_and_check(eg, dtype, q, k, v, dout, bias=(table(8, 4), 20, True))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_does_not_read_padding(eg, dtype):
    """What lies behind a sequence's length may hold anything."""
    q, k, v, dout = make(dtype, 3, 40, 90, 2, 2, 64, seed=11)
    ql, kl = [40, 17, 0], [90, 33, 65]
    want = run_and_check(eg, dtype, q, k, v, dout, q_lens=ql, k_lens=kl)
    for b in range(3):
        for t, n in ((q, ql[b]), (dout, ql[b]), (k, kl[b]), (v, kl[b])):
            t[b, n:] = float("nan")
        k[b, kl[b]::2] = float("inf")
    lens = [torch.tensor(n, dtype=torch.int32, device=DEV) for n in (ql, kl)]
    q, k, v, dout = (t.to(DEV) for t in (q, k, v, dout))
    out, lse = eg.attention(q, k, v, q_lens=lens[0], k_lens=lens[1])
    got = (out, lse, *eg.attention_backward(dout, q, k, v, out, lse, q_lens=lens[0], k_lens=lens[1])[:3])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hidden", [-math.inf, -3.4028234663852886e38, -1e30])
def test_attention_hidden_buckets(eg, dtype, hidden):
    """Table entries that hide their pairs: every key after the query; then everything for one head (its rows are empty)."""
    q, k, v, dout = make(dtype, 2, 77, 77, 3, 3, 32, seed=2)
    tab = table(16, 3)
    tab[8:] = hidden                                       # the upper half: keys after the query
    run_and_check(eg, dtype, q, k, v, dout, bias=(tab, 40, True))
    tab[:, 1] = hidden
    out, lse, dq, dk, dv, dtable = run_and_check(eg, dtype, q, k, v, dout, bias=(tab, 40, True))
    assert not out[:, :, 1].any() and torch.isneginf(lse[:, 1]).all() and not dq[:, :, 1].any() and not dk[:, :, 1].any()
    assert not dv[:, :, 1].any() and not dtable[:, 1].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_large_scores(eg, dtype):
    """Scores in the hundreds: rows that one key takes, and their gradients."""
    q, k, v, dout = make(dtype, 1, 100, 160, 2, 2, 64, seed=4, gain=4.0)
    run_and_check(eg, dtype, q, k, v, dout, scale=1.0)
    run_and_check(eg, dtype, q, k, v, dout, scale=-0.5, causal=True)
    run_and_check(eg, dtype, q, k, v, dout, scale=0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 40, 33, 128])
def test_attention_strides(eg, dtype, dim):
    """Slices of packed projections, head-major tensors, broadcast keys, odd offsets; gradients written into packed slices."""
    b, n, h = 2, 75, 3
    x = torch.randn(b, n, 3, h, dim, generator=torch.Generator().manual_seed(1)).to(T[dtype]).to(DEV)
    q, k, v = x.unbind(2)
    dout = torch.randn(b, h, n, dim, generator=torch.Generator().manual_seed(2)).to(T[dtype]).to(DEV).transpose(1, 2)
    packed = torch.full_like(x, 7.0)
    run_and_check(eg, dtype, q, k, v, dout, causal=True, grads=packed.unbind(2))
    head_major = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, k, v)]
    run_and_check(eg, dtype, *head_major, dout)
    run_and_check(eg, dtype, q, k[:1].expand(b, n, h, dim), v[:, :, :1].expand(b, n, h, dim), dout)
    room = torch.zeros(b * n * h * dim + 3, dtype=T[dtype], device=DEV)
    shifted = room[3:].view(b, n, h, dim)                   # 2- and 4-byte aligned only
    shifted.copy_(q)
    run_and_check(eg, dtype, shifted, k, v, dout, grads=(torch.empty(b * n * h * dim + 1, dtype=T[dtype], device=DEV)[1:].view(b, n, h, dim), None, None))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_empty_calls(eg, dtype):
    t = T[dtype]
    z = lambda *s: torch.zeros(s, dtype=t, device=DEV)  # noqa: E731
    tab = eg.PositionBias(table(8, 2).to(DEV), 20, True)
    for b, nq, nk in ((0, 4, 4), (2, 0, 4), (2, 4, 0), (0, 0, 0)):
        q, k, v = z(b, nq, 2, 16), z(b, nk, 2, 16), z(b, nk, 2, 16)
        out, lse = eg.attention(q, k, v, bias=tab)
        assert not out.any() and torch.isneginf(lse).all()
        dq, dk, dv, dtable = eg.attention_backward(q, q, k, v, out, lse, bias=tab)
        assert dtable.shape == (8, 2) and not any(x.any() for x in (dq, dk, dv, dtable))


@pytest.mark.gpu
def test_attention_beyond_32_bits(eg):
    """Keys, values and a gradient whose offsets pass 2^32 elements: tokens far apart in a long cache."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GiB")
    room = torch.zeros((1 << 32) + (1 << 20), dtype=torch.bfloat16, device=DEV)
    q, k, v, dout = make("bf16", 3, 5, 3, 2, 2, 64, seed=9)
    far, other = (room.as_strided((3, 3, 2, 64), (8192, (1 << 31) + 64, 128, 1), at) for at in (0, 1 << 19))
    far.copy_(k)
    run_and_check(eg, "bf16", q, far, v, dout, grads=(None, other, None))
    run_and_check(eg, "bf16", q, k, far, dout, grads=(None, None, other))
    del room, far, other


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_repeats_and_captures(eg, dtype):
    """The same bits every time: eager, on another stream, and in replays of a captured graph between eager calls."""
    q, k, v, dout = (t.to(DEV) for t in make(dtype, 2, 150, 190, 4, 2, 64, seed=8))
    lens = torch.tensor([190, 101], dtype=torch.int32, device=DEV)
    pb = eg.PositionBias(table(32, 4).to(DEV), 128, True)

    def step():
        out, lse = eg.attention(q, k, v, k_lens=lens, bias=pb)
        return (out, lse, *eg.attention_backward(dout, q, k, v, out, lse, k_lens=lens, bias=pb))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for n in range(4):
        for t in held:
            t.fill_(float("nan"))
        graph.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), n
        assert all(torch.equal(a, b) for a, b in zip(eager, want)), n
    # new inputs in the same memory: a replay reads them
    q.mul_(0.5)
    lens.copy_(torch.tensor([7, 190], dtype=torch.int32))
    graph.replay()
    want = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))


@pytest.mark.gpu
def test_attention_threads_and_shared_workspaces(eg):
    """Threads on streams of their own, and captured graphs that share one workspace and are replayed in order: the bits of a single call."""
    import threading
    calls = []
    for n, (dtype, shape, bias) in enumerate((("bf16", (130, 70, 40, 4, 4, 16), (16, 40)), ("bf16", (2, 300, 290, 4, 2, 64), (32, 128)), ("bf16", (1, 1, 5000, 8, 2, 128), None),
                                              ("f32", (3, 65, 200, 4, 4, 64), (8, 20)))):
        calls.append(([t.to(DEV) for t in make(dtype, *shape, seed=n)], bias and eg.PositionBias(table(bias[0], shape[3]).to(DEV), bias[1], True)))

    def step(call, ws=None):
        (q, k, v, dout), pb = call
        out, lse = eg.attention(q, k, v, causal=True, bias=pb, ws=ws)
        grads = eg.attention_backward(dout, q, k, v, out, lse, causal=True, bias=pb, ws=ws)
        return [out, lse, *(g for g in grads if g is not None)]

    want = [step(c) for c in calls]
    torch.cuda.synchronize()
    good = [0] * len(calls)

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(5):
                got = step(calls[i])
                stream.synchronize()
                good[i] += all(torch.equal(a, b) for a, b in zip(got, want[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert good == [5] * len(calls)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device=DEV)
    held = []
    for c in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(c, ws)
        held.append((graph, out))
    for _ in range(3):
        for _, out in held:
            for t in out:
                t.fill_(float("nan"))
        for graph, _ in held:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for (_, out), w in zip(held, want) for a, b in zip(out, w))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads_,nq,nk,offset,buckets,far,both", [
    (1, 1, 1, 0, 2, 2, False), (3, 77, 77, 0, 32, 128, True), (2, 300, 301, 0, 32, 128, True), (2, 301, 2051, 0, 32, 128, False), (4, 33, 500, 467, 20, 50, True),
    (2, 100, 9, -30, 8, 20, True), (1, 1200, 1300, 64, 4, 1024, True), (2, 1, 777, 776, 127, 1000, False), (5, 9, 4100, 2000, 128, 900, True)])
def test_position_bias(eg, dtype, heads_, nq, nk, offset, buckets, far, both):
    tab = table(buckets, heads_)
    pb = eg.PositionBias(tab.to(DEV), far, both)
    got = eg.position_bias(pb, nq, nk, offset=offset, dtype=T[dtype])
    want = ao.position_bias(tab.to(T[dtype]).double().numpy(), nq, nk, offset, far, both)
    assert np.array_equal(np64(got), want)
    rng = torch.Generator().manual_seed(nq + nk)
    for batch in (1, 3):
        d = torch.randn(batch, heads_, nq, nk, generator=rng).to(T[dtype])
        got = eg.position_bias_backward(d.to(DEV), pb, offset=offset)
        grad, size = ao.position_bias_backward(np64(d), buckets, offset, far, both)
        close(got, grad, (batch * 64 + nq + nk + 64) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(grad), "dtable")
        assert torch.equal(got, eg.position_bias_backward(d.to(DEV), pb, offset=offset))


@pytest.mark.gpu
def test_position_bias_empty(eg):
    pb = eg.PositionBias(table(8, 3).to(DEV), 20, True)
    assert eg.position_bias(pb, 0, 5).shape == (3, 0, 5) and eg.position_bias(pb, 5, 0).shape == (3, 5, 0)
    for s in ((0, 3, 4, 4), (2, 3, 0, 4), (2, 3, 4, 0)):
        assert not eg.position_bias_backward(torch.zeros(s, device=DEV), pb).any()


@pytest.mark.gpu
def test_bias_tensor_and_fused_bias_agree(eg):
    """The two ways to the table's gradient: in the attention's backward, and from the gradient of the bias as a tensor that an
    attention of elementary operations gives (fp32; both are within the oracle's bounds of fp64, twice that of each other)."""
    q, k, v, dout = (t.to(DEV) for t in make("f32", 2, 60, 90, 4, 4, 32, seed=12))
    pb = eg.PositionBias(table(16, 4).to(DEV), 40, True)
    out, lse = eg.attention(q, k, v, bias=pb)
    dtable = eg.attention_backward(dout, q, k, v, out, lse, bias=pb)[3]
    q2, k2, v2, do2 = (t.double().transpose(1, 2) for t in (q, k, v, dout))
    s = q2 @ k2.transpose(2, 3).contiguous() / math.sqrt(32) + eg.position_bias(pb, 60, 90).double()
    p = torch.softmax(s, -1)
    assert (p @ v2 - out.transpose(1, 2)).abs().max() < 1e-4
    ds = p * (do2 @ v2.transpose(2, 3).contiguous() - (do2 * (p @ v2)).sum(-1, keepdim=True))
    other = eg.position_bias_backward(ds.float().contiguous(), pb)
    want = ao.attention(np64(q), np64(k), np64(v), 1 / math.sqrt(32), bias=(np64(pb.table), 40, True), dout=np64(dout), saved=(np64(out), np64(lse)))
    close(dtable, want["dtable"], want["bound"]["dtable"], "fused")
    close(other, np64(dtable), 2 * want["bound"]["dtable"], "tensor")


@pytest.mark.gpu
def test_training_step_of_a_scored_layer(eg):
    """The operators as a training job uses them beside the evaluation: the attention block of an encoder layer runs forward and
    backward on a padded batch, its weights are stepped, and the layer's activations are scored before and after."""
    from paper_2201_06227_amd.evaluator import PlasticityEvaluator
    torch.manual_seed(3)
    b, n, h, d = 4, 48, 4, 16
    hid = h * d
    x = torch.randn(b, n, hid, device=DEV)
    w_in, w_out = torch.randn(3 * hid, hid, device=DEV) * hid ** -0.5, torch.randn(hid, hid, device=DEV) * hid ** -0.5
    tab = torch.randn(16, h, device=DEV) * 0.5
    lens = torch.tensor([48, 31, 1, 40], dtype=torch.int32, device=DEV)
    target = torch.randn(b, n, hid, device=DEV)
    live = (torch.arange(n, device=DEV)[None, :] < lens[:, None]).float()[..., None]

    def forward(w_in, w_out, tab):
        qkv = (x.view(-1, hid) @ w_in.t()).view(b, n, 3, h, d)
        pb = eg.PositionBias(tab, 30, True)
        out, lse = eg.attention(*qkv.unbind(2), q_lens=lens, k_lens=lens, bias=pb)
        y = (out.view(-1, hid) @ w_out.t()).view(b, n, hid) * live
        return qkv, pb, out, lse, y, 0.5 * ((y - target) * live).double().square().sum()

    qkv, pb, out, lse, y, loss = forward(w_in, w_out, tab)
    dy = ((y - target) * live).view(-1, hid)
    g_out = dy.t() @ out.view(-1, hid)
    dqkv = torch.empty_like(qkv)
    _, _, _, g_tab = eg.attention_backward((dy @ w_out).view(b, n, h, d), *qkv.unbind(2), out, lse, q_lens=lens, k_lens=lens, bias=pb,
                                           dq=dqkv[:, :, 0], dk=dqkv[:, :, 1], dv=dqkv[:, :, 2])
    g_in = dqkv.view(-1, 3 * hid).t() @ x.view(-1, hid)
    for name, g in (("w_in", g_in), ("w_out", g_out), ("tab", g_tab)):
        step = torch.randn_like(g)
        arg = dict(w_in=w_in, w_out=w_out, tab=tab)
        at = lambda e: forward(**{**arg, name: arg[name] + e * step})[5].item()  # noqa: E731
        diff, want = (at(2e-3) - at(-2e-3)) / 4e-3, (g.double() * step.double()).sum().item()
        # the difference quotient's own error: third order in the step, and the loss's fp32 noise over it
        assert abs(diff - want) < 2e-2 * abs(want) + 1e-5 * loss.item() / 4e-3, (name, diff, want)
    ev = PlasticityEvaluator(eg.FC_RELU, dict(batch=b, c_in=n * hid, c_out=hid), [torch.randn(hid, n * hid, device=DEV) * 0.02], [None], device=DEV)
    p = [ev.step(out.reshape(b, -1).contiguous(), [torch.relu(out.reshape(b, -1) @ torch.randn(n * hid, hid, device=DEV))]).item() for _ in range(2)]
    assert all(math.isfinite(v) and v > 0 for v in p)
