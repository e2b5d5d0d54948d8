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
