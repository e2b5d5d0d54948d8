"""Attention of the training model at the ends of its ranges: values that are not finite, kernels that only large calls reach, arguments at
their limits.  Against the fp64 oracle's bounds, or exactly where the numbers are whole."""
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from test_attention import DEV, STEPS, T, close, eg, make, np64, run_and_check  # noqa: F401  (eg: the fixture)

# A call for each way through the forward pass: a workgroup of four waves for a few rows with one, four and twenty workgroups to
# share the keys, and tiles of 128 queries (at least 48 of them).  batch, q_len, k_len, heads, kv_heads, dim
WAYS = {"few": (2, 3, 200, 4, 2, 64), "four splits": (2, 1, 900, 4, 2, 64), "twenty splits": (1, 1, 5000, 8, 2, 128), "tiles": (4, 130, 200, 12, 4, 64)}


def clean(dtype, q, k, v, **how):
    h_out, h_op = STEPS[dtype]
    scale = np.float64(np.float32(1.0 / math.sqrt(q.shape[3])))
    return ao.attention(np64(q), np64(k), np64(v), scale, half_step=h_out, operand_step=h_op, **how)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("way", WAYS)
def test_a_query_that_is_nan(eg, dtype, way):  # noqa: F811
    """Its row is NaN and no other: an empty row's zeros would hide it."""
    q, k, v, _ = make(dtype, *WAYS[way], seed=21)
    want = clean(dtype, q, k, v)
    b, i, h = q.shape[0] - 1, q.shape[1] - 1, 3
    q[b, i, h, 5] = math.nan
    out, _ = eg.attention(q.to(DEV), k.to(DEV), v.to(DEV))
    assert torch.isnan(out[b, i, h]).all()
    want["out"][b, i, h], out[b, i, h] = 0.0, 0.0
    close(out, want["out"], want["bound"]["out"], way)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("at", [0, 0.5, 1])
def test_a_value_that_is_not_finite(eg, dtype, way, at):  # noqa: F811
    """Every query that sees it has it in its feature, with its sign, and nowhere else."""
    q, k, v, _ = make(dtype, *WAYS[way], seed=22)
    want = clean(dtype, q, k, v)["out"]
    j, g, group = int(at * (k.shape[1] - 1)), v.shape[2] - 1, q.shape[2] // v.shape[2]
    rows = (0, slice(None), slice(g * group, (g + 1) * group))
    for x in (math.inf, -math.inf, math.nan):
        v[0, j, g, 7] = x
        out, _ = eg.attention(q.to(DEV), k.to(DEV), v.to(DEV))
        got = np64(out)
        assert np.array_equal(got[rows][..., 7], np.full_like(want[rows][..., 7], x), equal_nan=True), x
        got[rows][..., 7] = 0.0
        assert np.isfinite(got).all(), x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("way", WAYS)
def test_log_sum_exp_of_scores_that_are_not_finite(eg, dtype, way):  # noqa: F811
    """NaN where a score is NaN or overflows; minus infinity is that of a row without a visible pair."""
    q, k, v, _ = make(dtype, *WAYS[way], seed=23)
    lens = [k.shape[1]] * (q.shape[0] - 1) + [0 if q.shape[0] > 1 else k.shape[1]]
    kl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = clean(dtype, q, k, v, k_lens=lens)
    group, j = q.shape[2] // k.shape[2], k.shape[1] // 2
    nan_q, nan_k, big_q, big_k = q.clone(), k.clone(), q.clone(), k.clone()
    nan_q[0, 0, 1, 3] = math.nan
    nan_k[0, j, 1, 3] = math.nan
    big_q[0, 0, group, 3], big_k[0, j, 1, 3] = 2.0 ** 70, 2.0 ** 70     # of head `group`, the first of key head 1
    big_q[0, :, group + 1:2 * group, 3] = 0.0
    big_q[0, 1:, group, 3] = 0.0
    for what, (qq, kk), rows in (("query", (nan_q, k), (0, 1, 0)), ("key", (q, nan_k), (0, slice(group, 2 * group))), ("overflow", (big_q, big_k), (0, group, 0))):
        out, lse = eg.attention(qq.to(DEV), kk.to(DEV), v.to(DEV), k_lens=kl)
        assert torch.isnan(lse[rows]).all() and torch.isnan(out.transpose(1, 2)[rows]).all(), what
        if what != "overflow":                                 # (there the other rows are others too)
            lse[rows] = 0.0
            exp = want["lse"].copy()
            exp[rows] = 0.0
            close(lse, exp, want["bound"]["lse"], what)
        else:
            assert torch.isnan(lse).sum() == 1
        if lens[-1] == 0:
            assert torch.isneginf(lse[-1]).all() and not out[-1].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 70, 150, 4, 2, 64), (1, 150, 300, 4, 2, 128), (64, 20, 40, 4, 2, 32), (64, 70, 200, 4, 2, 64)], ids=str)
def test_gradients_of_a_query_that_is_nan(eg, dtype, shape):  # noqa: F811
    """Its own gradient, those of the keys and values it sees and of its head's table are NaN; everything else is as without it."""
    q, k, v, dout = make(dtype, *shape, seed=24)
    b, i, h, g = shape[0] - 1, 11, 3, 1
    tab = torch.randn(8, 4, generator=torch.Generator().manual_seed(1))
    q[b, i, h, 2] = math.nan
    on = [t.to(DEV) for t in (q, k, v)]
    pb = eg.PositionBias(tab.to(DEV), 20, True)
    out, lse = eg.attention(*on, bias=pb)
    dq, dk, dv, dtable = eg.attention_backward(dout.to(DEV), *on, out, lse, bias=pb)
    assert torch.isnan(dq[b, i, h]).all() and torch.isnan(dk[b, :, g]).all() and torch.isnan(dv[b, :, g]).all()
    assert torch.isnan(dtable[[n for n in range(8) if n != 4], h]).all()        # (row 4 would be distance 0 of the later keys, which the earlier ones have)
    saved, h_out, h_op = (np64(out), np64(lse)), *STEPS[dtype]
    saved[0][b, i, h], saved[1][b, h, i] = 0.0, -math.inf
    q[b, i, h, 2] = 0.0
    want = ao.attention(np64(q), np64(k), np64(v), np.float64(np.float32(1.0 / math.sqrt(shape[5]))), bias=(np64(tab), 20, True), dout=np64(dout), saved=saved,
                        half_step=h_out, operand_step=h_op)
    for name, t, at in (("dq", dq, (b, i, h)), ("dk", dk, (b, slice(None), g)), ("dv", dv, (b, slice(None), g)), ("dtable", dtable, (slice(None), h))):
        t[at] = 0.0
        want[name][at] = 0.0
        close(t, want[name], want["bound"][name], name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("x", [math.nan, math.inf])
@pytest.mark.parametrize("shape", [(2, 20, 200, 4, 2, 64), (2, 9, 900, 4, 2, 64), (4, 130, 200, 12, 4, 64), (64, 70, 40, 4, 2, 64), (33, 100, 200, 4, 4, 33)], ids=str)
def test_rows_without_a_pair_are_zero_beside_values_that_are_not_finite(eg, dtype, x, shape):  # noqa: F811
    """Queries behind their sequence, and causal ones before its first key: zeros in out and dq, whatever the keys and values of their sequence hold."""
    nq, nk = shape[1], shape[2]
    tab = eg.PositionBias(torch.randn(8, shape[3], generator=torch.Generator().manual_seed(2)).to(DEV), 20, True)
    for causal, ql, kl in ((False, nq - 3, nk - 5), (True, nq - 3, nk - 5), (True, nq - 1, 4), (True, nq, 1)):
        q, k, v, dout = (t.to(DEV) for t in make(dtype, *shape, seed=25))
        k[0, 0, 0, 1] = v[0, 0, 1, 1] = x
        lens = [torch.full((shape[0],), n, dtype=torch.int32, device=DEV) for n in (ql, kl)]
        none = [i for i in range(nq) if i >= ql or (causal and i + kl - ql < 0)]
        for pb in (None, tab):
            how = dict(causal=causal, q_lens=lens[0], k_lens=lens[1], bias=pb)
            out, lse = eg.attention(q, k, v, **how)
            dq, dk, dv, _ = eg.attention_backward(dout, q, k, v, out, lse, **how)
            what = (causal, ql, kl, pb is not None)
            assert (out[:, none] == 0).all() and torch.isneginf(lse[:, :, none]).all(), what
            assert (dq[:, none] == 0).all(), what
            assert (dk[:, kl:] == 0).all() and (dv[:, kl:] == 0).all(), what
            assert torch.isfinite(out[1:]).all() and all(torch.isfinite(t[1:]).all() for t in (dq, dk, dv)), what


def test_no_silent_loss_of_a_graph(eg):  # noqa: F811
    """The calls record nothing for autograd, so they refuse tensors that want a gradient through them (before anything else: on the host)."""
    x, tab = torch.zeros(1, 2, 2, 8), torch.zeros(8, 2)
    want, bias = x.clone().requires_grad_(), eg.PositionBias(tab.clone().requires_grad_(), 20)
    calls = [lambda: eg.attention(want, x, x), lambda: eg.attention(x, want, x), lambda: eg.attention(x, x, want), lambda: eg.attention(x, x, x, bias=bias),
             lambda: eg.attention_backward(want, x, x, x, x, x), lambda: eg.position_bias(bias, 4, 4),
             lambda: eg.position_bias_backward(torch.zeros(1, 2, 4, 4, requires_grad=True), eg.PositionBias(tab, 20))]
    for call in calls:
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="device"):       # (host tensors)
            call()
    with pytest.raises(ValueError, match="device"):                            # what a hand-written backward pass has saved may require one
        eg.attention_backward(x, want, want, want, want, x, bias=bias)


@pytest.mark.gpu
def test_calls_of_an_autograd_function(eg):  # noqa: F811
    """In a torch.autograd.Function, where there is no graph, leaves may require gradients; they get those of the formula."""
    q, k, v, dout = (t.to(DEV) for t in make("f32", 2, 20, 30, 4, 2, 16, seed=31))
    tab = torch.randn(8, 4, generator=torch.Generator().manual_seed(3)).to(DEV)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, tab):
            out, lse = eg.attention(q, k, v, bias=eg.PositionBias(tab, 20))
            ctx.save_for_backward(q, k, v, tab, out, lse)
            return out

        @staticmethod
        def backward(ctx, dout):
            q, k, v, tab, out, lse = ctx.saved_tensors
            return eg.attention_backward(dout, q, k, v, out, lse, bias=eg.PositionBias(tab, 20))

    leaves = [t.clone().requires_grad_() for t in (q, k, v, tab)]
    Attention.apply(*leaves).backward(dout)
    out, lse = eg.attention(q, k, v, bias=eg.PositionBias(tab, 20))
    for leaf, g in zip(leaves, eg.attention_backward(dout, q, k, v, out, lse, bias=eg.PositionBias(tab, 20))):
        assert torch.equal(leaf.grad, g)


@pytest.mark.parametrize("shape", [(1, 2, (1 << 32) + 4, 1), ((1 << 32) + 2, 2, 1, 1), (1, 2, 1, (1 << 32) + 1)])
def test_sizes_beyond_c(eg, monkeypatch, shape):  # noqa: F811
    """A bias gradient with a size that a C int does not hold is refused, not taken for the size that is left of it (tensors without memory)."""
    monkeypatch.setattr(eg, "_same_device", lambda *t: 0)
    monkeypatch.setattr(eg, "_dev", lambda t: t)
    with pytest.raises(ValueError, match="out of range"):
        eg.position_bias_backward(torch.empty(shape, device="meta"), eg.PositionBias(torch.zeros(8, 2), 20))
    with pytest.raises(ValueError, match="out of range"):
        eg.PositionBias(torch.empty((1 << 32) + 8, 1, device="meta"), 20).c_struct()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("strides", [(40, 1, 20, 1), (40, 8, 1, 1), (0, 1, 0, 1), (0, 0, 0, 1)], ids=str)
def test_inputs_whose_elements_overlap(eg, dtype, strides):  # noqa: F811
    """Windows of one run of values, broadcast heads, tokens and sequences: any strides whose features are contiguous."""
    shape = (2, 3, 2, 8)
    x = torch.randn(4, 100, generator=torch.Generator().manual_seed(5)).to(T[dtype]).to(DEV)
    run_and_check(eg, dtype, *(r.as_strided(shape, strides) for r in x))


def test_workspaces_that_are_smaller_than_they_look(eg, monkeypatch):  # noqa: F811
    """A workspace whose elements lie on each other has fewer bytes than elements: refused on the host (where these tensors are)."""
    monkeypatch.setattr(eg, "_same_device", lambda *t: 0)
    monkeypatch.setattr(eg, "_dev", lambda t: t)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    monkeypatch.setattr(eg, "_stream", lambda: 0)
    x, ws, pb = torch.zeros(1, 2, 2, 8), torch.zeros(256, dtype=torch.uint8)[:1].expand(1 << 20), eg.PositionBias(torch.zeros(8, 2), 20)
    lse = torch.zeros(1, 2, 2)
    for call in (lambda: eg.attention(x, x, x, ws=ws), lambda: eg.attention_backward(x, x, x, x, x, lse, ws=ws), lambda: eg.position_bias_backward(torch.zeros(1, 2, 4, 4), pb, ws=ws)):
        with pytest.raises(ValueError, match="workspace"):
            call()


@pytest.mark.gpu
def test_eight_million_sequences(eg):  # noqa: F811
    """2^23 workgroups of 256 threads are half of what a launch holds: sequences of one token, whose probability is 1."""
    n = 1 << 23
    q, k, v, dout = (torch.randn(n, 1, 1, 1, device=DEV, generator=torch.Generator(DEV).manual_seed(i)).bfloat16() for i in range(4))
    out, lse = eg.attention(q, k, v)
    assert torch.equal(out, v)
    score = q.float() * k.float()                         # exact: two factors of 8 bits
    assert ((lse.view(-1) - score.view(-1)).abs() <= 4 * 2.0 ** -24 * score.view(-1).abs()).all()      # to base 2 and back: two products and two constants
    dq, dk, dv, _ = eg.attention_backward(dout, q, k, v, out, lse)
    # p = 1 within the error of lse and of the exponent's two roundings, far below half a step of bf16 (2^-8): p is 1; ds = p (dout v - dout out) = 0
    assert torch.equal(dv, dout) and not dq.any() and not dk.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2, 70, 200, 4, 4, 64), (64, 40, 70, 4, 4, 64), (64, 40, 200, 4, 4, 64)], ids=str)
@pytest.mark.parametrize("offset", [-1e9, 1e9, -3e9, -1e10, 1e10, -9e29])
def test_an_offset_of_a_whole_head(eg, dtype, shape, offset):  # noqa: F811
    """A table entry that is large, but hides nothing, for all pairs of a head: an fp32 log-sum-exp has no bits left for its probabilities, but its
    numbers stay finite, and the other heads' are what they are without it."""
    tab = torch.randn(8, 4, generator=torch.Generator().manual_seed(6))
    q, k, v, dout = make(dtype, *shape, seed=33)
    run_and_check(eg, dtype, q, k, v, dout, bias=(tab, 20, True))
    on = [t.to(DEV) for t in (q, k, v, dout)]
    results = []
    for x in (tab[:, 1].clone(), offset):
        tab[:, 1] = x
        pb = eg.PositionBias(tab.to(DEV), 20, True)
        out, lse = eg.attention(*on[:3], bias=pb)
        dq, dk, dv, dtable = eg.attention_backward(on[3], *on[:3], out, lse, bias=pb)
        results.append((out, lse.transpose(1, 2), dq, dk, dv, dtable[:, :, None].transpose(0, 1)[None].transpose(1, 2)))
    rest = [0, 2, 3]
    for a, b in zip(*results):
        assert torch.equal(a[:, :, rest], b[:, :, rest])
    # scores of this head are below 6.5 in size, so p < 666 whatever part of them is left; |dP - D| < 2 * 64 * 25; at most 200 keys of size 5, scale 1/8
    for name, t in zip(("out", "dq", "dk", "dv"), (results[1][n] for n in (0, 2, 3, 4))):
        assert torch.isfinite(t).all() and t.abs().max() < 666 * 3200 * 200 * 5 / 8, name
    assert torch.isfinite(results[1][5]).all()


# Calls of at least 48 tiles of 128 queries, which go to the kernel for whole tiles whatever their keys are; several tiles of keys.
TILES = [(4, 130, 200, 12, 4, 96), (4, 130, 600, 12, 12, 128), (4, 130, 330, 12, 6, 127), (2, 257, 520, 9, 3, 128), (4, 129, 641, 12, 3, 64), (8, 140, 300, 6, 2, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", TILES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("kind", ["plain", "causal", "bias", "causal bias lengths"])
def test_whole_tiles(eg, dtype, shape, kind):  # noqa: F811
    b, nq, nk, h = shape[:4]
    bias = (torch.randn(32, h, generator=torch.Generator().manual_seed(7)), 128, "causal" not in kind) if "bias" in kind else None
    rng = np.random.default_rng(nk)
    lens = dict(q_lens=[nq, *rng.integers(1, nq + 1, b - 1).tolist()], k_lens=[nk, *rng.integers(1, nk + 1, b - 1).tolist()]) if "lengths" in kind else {}
    run_and_check(eg, dtype, *make(dtype, *shape, seed=nk), causal="causal" in kind, bias=bias, **lens)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(4, 130, 330, 12, 4, 128), (64, 70, 40, 4, 2, 64), (64, 40, 200, 4, 2, 33)], ids=str)
@pytest.mark.parametrize("causal", [False, True])
def test_padding_of_large_calls_is_not_read(eg, dtype, shape, causal):  # noqa: F811
    """What lies behind a sequence's length, NaN and infinity among it, in the kernel for whole tiles and the backward pass of few keys."""
    b, nq, nk = shape[:3]
    q, k, v, dout = make(dtype, *shape, seed=41)
    rng = np.random.default_rng(b)
    ql, kl = rng.integers(0, nq + 1, b).tolist(), rng.integers(0, nk + 1, b).tolist()
    want = run_and_check(eg, dtype, q, k, v, dout, causal=causal, q_lens=ql, k_lens=kl)
    for i in range(b):
        for t, n in ((q, ql[i]), (dout, ql[i]), (k, kl[i]), (v, kl[i])):
            t[i, n:] = math.nan
        k[i, kl[i]::2] = math.inf
    lens = [torch.tensor(n, dtype=torch.int32, device=DEV) for n in (ql, kl)]
    q, k, v, dout = (t.to(DEV) for t in (q, k, v, dout))
    out, lse = eg.attention(q, k, v, causal=causal, q_lens=lens[0], k_lens=lens[1])
    got = (out, lse, *eg.attention_backward(dout, q, k, v, out, lse, causal=causal, q_lens=lens[0], k_lens=lens[1])[:3])
    for a, w in zip(got, want):
        assert torch.equal(a, w)


def whole(rng, *shape, most=1):
    """Whole numbers in [-most, most], none of them 0."""
    x = torch.randint(1, most + 1, shape, generator=rng) * (2 * torch.randint(0, 2, shape, generator=rng) - 1)
    return x.double()


COUNTS = {**WAYS, "heads of 128": (2, 140, 300, 16, 4, 128), "odd rows": (2, 70, 300, 4, 2, 75), "few keys": (64, 70, 100, 4, 2, 64), "keys of eight waves": (33, 90, 256, 4, 4, 40),
          "short": (2, 33, 65, 2, 1, 16)}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("way", COUNTS)
@pytest.mark.parametrize("causal", [False, True])
def test_every_pair_counts_once(eg, dtype, way, causal):  # noqa: F811
    """All scores 0 (queries, or keys, of 0), whole numbers elsewhere: out is a mean of whole numbers and every gradient a sum of whole numbers over a
    number of keys, so that one pair too few or too many shows where a bound for ordinary numbers would let it pass.
    Bounds: p is 1 in the forward pass, exactly; sums of whole numbers are exact; a division and a product are left, 2 u.  Backward, L = log n < 9 with
    4 roundings and the exponent's: p is off by less than (5 * 9 + 16) u < 2^-18 of itself, a sum of n terms by n u; bf16 rounds p where it enters a
    product, by 2^-8 of itself at most and not at all where n is a power of two, which the lengths are without the causal mask."""
    b, nq, nk, h, g, d = COUNTS[way]
    rng = torch.Generator().manual_seed(51)
    lens = [1 << (nk.bit_length() - 1 - i % 4) for i in range(b)]
    ql = [nq - i % 3 for i in range(b)]
    kl, qls = (torch.tensor(n, dtype=torch.int32, device=DEV) for n in (lens, ql))
    v, dout = whole(rng, b, nk, g, d, most=8), whole(rng, b, nq, h, d)
    tab = torch.zeros(16, h)
    u, half, operand = 2.0 ** -24, *STEPS[dtype]
    if not causal:
        operand = 0.0
    zero_k = dict(q=whole(rng, b, nq, h, d, most=4), k=torch.zeros(b, nk, g, d).double())
    zero_q = dict(q=torch.zeros(b, nq, h, d).double(), k=whole(rng, b, nk, g, d, most=4))
    for x in (zero_k, zero_q):
        on = [t.to(T[dtype]).to(DEV) for t in (x["q"], x["k"], v)]
        pb = eg.PositionBias(tab.to(DEV), 40, not causal)
        out, lse = eg.attention(*on, causal=causal, q_lens=qls, k_lens=kl, scale=0.5, bias=pb)
        bare = eg.attention(*on, causal=causal, q_lens=qls, k_lens=kl, scale=0.5)[0]
        # the gradients' own inputs: values of 1 and -1 and a saved output of 0, so that dS is a whole number <= d over a number of keys
        ones = torch.sign(v)
        saved = torch.zeros_like(out)
        grads = eg.attention_backward(dout.to(T[dtype]).to(DEV), *on[:2], ones.to(T[dtype]).to(DEV), saved, lse, causal=causal, q_lens=qls, k_lens=kl, scale=0.5, bias=pb)
        want, bound = [np.zeros(s.shape) for s in (x["q"], x["q"], x["k"], x["k"], tab)], [np.zeros(s.shape) for s in (x["q"], x["q"], x["k"], x["k"], tab)]
        for i in range(b):
            n, m = ql[i], lens[i]
            shift = m - n if causal else 0
            seen = (np.arange(m)[None] <= np.arange(n)[:, None] + shift) if causal else np.ones((n, m), bool)
            p = seen / np.maximum(seen.sum(1, keepdims=True), 1)
            grid = ao.bucket_grid(n, m, shift, 16, 40, not causal)
            for j in range(h):
                e = j // (h // g)
                vv, ov, do, qq, kk = (np64(t) for t in (v[i, :m, e], ones[i, :m, e], dout[i, :n, j], x["q"][i, :n, j], x["k"][i, :m, e]))
                want[0][i, :n, j] = (seen @ vv) / np.maximum(seen.sum(1, keepdims=True), 1)        # (the sum first: it is whole)
                bound[0][i, :n, j] = (half + 2 * u) * np.abs(want[0][i, :n, j])
                ds = p * (do @ ov.T)
                rel = 2.0 ** -18 + operand
                want[1][i, :n, j] = 0.5 * ds @ kk
                bound[1][i, :n, j] = 0.5 * np.abs(ds) @ np.abs(kk) * (rel + m * u)
                want[2][i, :m, e] += 0.5 * ds.T @ qq
                bound[2][i, :m, e] += 0.5 * np.abs(ds).T @ np.abs(qq) * (rel + n * h // g * u)
                want[3][i, :m, e] += p.T @ do
                bound[3][i, :m, e] += p.T @ np.abs(do) * (rel + n * h // g * u)
                want[4][:, j] += np.bincount(grid.ravel(), weights=ds.ravel(), minlength=16)
                bound[4][:, j] += np.bincount(grid.ravel(), weights=np.abs(ds).ravel(), minlength=16) * (2.0 ** -18 + (n + m) * u)
        for at in (1, 2, 3):
            bound[at] += half * np.abs(want[at])
        close(out, want[0], bound[0], "out")
        assert torch.equal(out, bare)
        for name, t, w, e in zip(("dq", "dk", "dv", "dtable"), grads, want[1:], bound[1:]):
            close(t, w, e, name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 1, 301, 2051), (5, 3, 77, 77), (1, 1, 1201, 1301), (7, 2, 33, 4099), (2, 3, 130, 2048), (40, 1, 9, 1), (1, 1, 1, 1), (2, 2, 260, 264), (9, 1, 8, 8195)], ids=str)
@pytest.mark.parametrize("offset,buckets,far,both", [(0, 32, 128, True), (7, 2, 2, False), (100, 128, 1000, False)])
def test_every_bias_gradient_counts_once(eg, dtype, shape, offset, buckets, far, both):  # noqa: F811
    """Whole numbers up to 3, whose sums stay below 2^24: every partial sum is exact in fp32, so the result is."""
    d = whole(torch.Generator().manual_seed(sum(shape)), *shape, most=3)
    grad, size = ao.position_bias_backward(d.numpy(), buckets, offset, far, both)
    assert size.max() < 2 ** 24
    got = eg.position_bias_backward(d.to(T[dtype]).to(DEV), eg.PositionBias(torch.zeros(buckets, shape[1], device=DEV), far, both), offset=offset)
    assert np.array_equal(np64(got), grad)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 16, 1100, 2101), (2, 4, 4110, 4128)], ids=str)
def test_bias_of_many_columns_to_a_workgroup(eg, dtype, shape):  # noqa: F811
    """Rows enough for workgroups that go through several pieces of the columns: the bias as a tensor, and whole numbers' sums, exactly."""
    b, h, nq, nk = shape
    offset, buckets, far = 50, 32, 128
    rel = np.arange(-nq + 1 - offset, nk - offset)
    by = np.array([ao.bucket_of(int(r), buckets, far, True) for r in rel])
    grid = by[np.arange(nk)[None, :] - np.arange(nq)[:, None] + nq - 1]
    tab = torch.randn(buckets, h, generator=torch.Generator().manual_seed(8))
    pb = eg.PositionBias(tab.to(DEV), far, True)
    got = eg.position_bias(pb, nq, nk, offset=offset, dtype=T[dtype])
    want = tab.to(T[dtype]).to(DEV)[torch.from_numpy(grid).to(DEV)].permute(2, 0, 1)
    assert torch.equal(got, want)
    d = torch.randint(-1, 2, shape, generator=torch.Generator().manual_seed(9), dtype=torch.int8)
    got = eg.position_bias_backward(d.to(DEV).to(T[dtype]), pb, offset=offset)
    sums = np.stack([np.bincount(grid.ravel(), weights=d[:, k].sum(0, dtype=torch.int64).numpy().ravel(), minlength=buckets) for k in range(h)], 1)
    assert np.abs(sums).max() < 2 ** 22 and np.array_equal(np64(got), sums)      # (partial sums of random signs: thousands, far below 2^24)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what,x", [("key", math.nan), ("value", math.nan), ("value", math.inf)])
@pytest.mark.parametrize("shape", [(2, 70, 150, 4, 2, 64), (1, 150, 300, 4, 2, 128), (64, 20, 40, 4, 2, 32), (64, 70, 200, 4, 2, 64)], ids=str)
def test_gradients_of_a_key_or_value_that_is_not_finite(eg, dtype, what, x, shape):  # noqa: F811
    """No gradient of the heads that see it is finite, but dv beside a value (which it does not depend on); all others are as without it."""
    q, k, v, dout = make(dtype, *shape, seed=26)
    h, nk = shape[3], shape[2]
    tab = torch.randn(8, h, generator=torch.Generator().manual_seed(4))
    pb = eg.PositionBias(tab.to(DEV), 20, True)
    scale = np.float64(np.float32(1.0 / math.sqrt(shape[5])))
    out, lse = eg.attention(*(t.to(DEV) for t in (q, k, v)), bias=pb)
    want = ao.attention(np64(q), np64(k), np64(v), scale, bias=(np64(tab), 20, True), dout=np64(dout), saved=(np64(out), np64(lse)), half_step=STEPS[dtype][0],
                        operand_step=STEPS[dtype][1])
    (k if what == "key" else v)[0, nk // 2, 1, 5] = x
    on = [t.to(DEV) for t in (q, k, v)]
    out, lse = eg.attention(*on, bias=pb)
    dq, dk, dv, dtable = eg.attention_backward(dout.to(DEV), *on, out, lse, bias=pb)
    heads = slice(h // 2, h)
    for name, t, at in (("dq", dq, (0, slice(None), heads)), ("dk", dk, (0, slice(None), 1)), ("dv", dv, (0, slice(None), 1)), ("dtable", dtable, (slice(None), heads))):
        if name == "dv" and what == "value":
            at = None
        elif name != "dtable":
            assert not torch.isfinite(t[at]).any(), name
        if at is not None:
            t[at] = 0.0
            want[name][at] = 0.0
        close(t, want[name], want["bound"][name], name)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,causal", [((1, 1, 700, 64, 1, 128), True), ((1, 1, 700, 33, 1, 128), False), ((2, 3, 200, 64, 2, 64), False), ((1, 200, 900, 4, 2, 128), False),
                                          ((4, 130, 400, 12, 3, 96), False), ((130, 40, 200, 2, 1, 64), False), ((64, 30, 100, 2, 2, 32), True)], ids=str)
def test_the_largest_tables(eg, dtype, shape, causal):  # noqa: F811
    """128 buckets up to distances beyond 900 on both sides, and up to 64 query heads to a key head: the most LDS that a call takes."""
    run_and_check(eg, dtype, *make(dtype, *shape, seed=61), causal=causal, bias=(torch.randn(128, shape[3], generator=torch.Generator().manual_seed(9)), 1024, True))
    run_and_check(eg, dtype, *make(dtype, *shape, seed=62), causal=causal, bias=(torch.randn(127, shape[3], generator=torch.Generator().manual_seed(10)), 1024, False))


@pytest.mark.gpu
@pytest.mark.parametrize("kw", [dict(b=4, s=48, hidden=128, heads=4, ffn=256, n_layers=2), dict(b=3, s=33, hidden=96, heads=3, ffn=160, n_layers=1)], ids=str)
def test_training_and_scoring_of_encoder_layers(eg, orc, kw):  # noqa: F811
    """An encoder in training whose attention is this one, and the evaluation of its layers: the activations that the training forward leaves are scored
    against the int8 reference of a snapshot of the same layers, before and after a step along the gradients."""
    import torch.nn.functional as F

    import synth_inputs as si
    from paper_2201_06227_amd.evaluator import PlasticityEvaluator
    wl = si.make_bert(seed=77, train_act_dtype="f32", **kw)
    hid, nh, n_layers = kw["hidden"], kw["heads"], kw["n_layers"]

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, qkv):
            out, lse = eg.attention(*qkv.unbind(2))
            ctx.save_for_backward(qkv, out, lse)
            return out

        @staticmethod
        def backward(ctx, dout):
            qkv, out, lse = ctx.saved_tensors
            dqkv = torch.empty_like(qkv)
            eg.attention_backward(dout, *qkv.unbind(2), out, lse, dq=dqkv[:, :, 0], dk=dqkv[:, :, 1], dv=dqkv[:, :, 2])
            return dqkv

    def plain(qkv):
        q, k, v = (t.transpose(1, 2) for t in qkv.unbind(2))
        return (torch.softmax(q @ k.transpose(2, 3) / math.sqrt(hid // nh), -1) @ v).transpose(1, 2)

    def forward(x, weights, attend):
        acts = []
        for l in range(n_layers):
            wq, wo, w1, w2 = weights[4 * l:4 * l + 4]
            b, s = x.shape[:2]
            y = F.layer_norm(x + attend(F.linear(x, wq).view(b, s, 3, nh, hid // nh)).reshape(b, s, hid) @ wo.t(), (hid,), eps=1e-12)
            x = F.layer_norm(y + F.linear(F.gelu(F.linear(y, w1)), w2), (hid,), eps=1e-12)
            acts.append(x)
        return acts

    x, target = torch.from_numpy(wl.x), torch.randn(wl.x.shape, generator=torch.Generator().manual_seed(1))

    def run(dtype, dev, attend):
        w = [torch.from_numpy(t).to(dev, dtype).requires_grad_() for t in wl.train_weights]
        acts = forward(x.to(dev, dtype), w, attend)
        (0.5 * (acts[-1] - target.to(dev, dtype)).square().sum()).backward()
        return w, acts

    w, acts = run(torch.float32, DEV, Attention.apply)
    w64, acts64 = run(torch.float64, "cpu", plain)
    # fp32 sums of at most 288 terms, a dozen one behind the other: 12 * 290 u = 2e-4 of the terms' size, and terms that cancel to a fifth of it
    for a, b in zip([*acts, *(t.grad for t in w)], [*acts64, *(t.grad for t in w64)]):
        a, b = a.detach().double().cpu(), b.detach()
        assert (a - b).norm() <= 1e-3 * b.norm()
    ev = PlasticityEvaluator(wl.kind, wl.dims, [torch.from_numpy(t).to(DEV) for t in wl.weights], [None] * len(wl.weights), device=DEV)
    wl.biases = [None] * len(wl.weights)
    a_ref = orc.ref_forward(wl)["a_ref"]
    with torch.no_grad():
        stepped = forward(x.to(DEV), [t - 1e-3 * t.grad for t in w], lambda qkv: eg.attention(*qkv.unbind(2))[0])
    for hooked in (acts, stepped):
        a_t = [a.detach().reshape(a.shape[0], -1).contiguous() for a in hooked]
        p = ev.step(x.to(DEV), a_t).cpu().numpy()
        for l, t in enumerate(a_t):
            want = orc.sp_loss(t.cpu().numpy(), a_ref[l].reshape(t.shape))
            assert abs(p[l] - want) <= 1e-4 * abs(want) + 1e-12 * 4.0 / kw["b"], l


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [-5000, 5000])
def test_far_sums_that_cancel(eg, dtype, offset):  # noqa: F811
    """Score gradients beyond the table, all of one bucket, whose large parts cancel next to each other: what is left is the sum, not the rounding of fp32."""
    d = torch.zeros(2, 3, 64, 640)
    d[:, :, ::8, 0::8], d[:, :, ::8, 1::8], d[:, :, ::8, 2::8] = 2.0 ** 25, 1.0, -2.0 ** 25
    pb = eg.PositionBias(torch.zeros(32, 3, device=DEV), 128, True)
    got = eg.position_bias_backward(d.to(T[dtype]).to(DEV), pb, offset=offset)
    want = torch.zeros(32, 3)
    want[31 if offset < 0 else 15] = 2 * 8 * 80
    assert torch.equal(got.cpu(), want)
