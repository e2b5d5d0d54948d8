"""Attention of the training model at the ends of its ranges: values that are not finite, kernels that only large calls reach, arguments at
their limits.  Against the fp64 oracle's bounds, or exactly where the numbers are whole."""
import math

import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao
from test_attention import DEV, STEPS, T, close, eg, make, np64  # noqa: F401  (eg: the fixture)

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
