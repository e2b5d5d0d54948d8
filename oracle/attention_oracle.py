"""Attention with a learned relative position bias and its gradients in fp64 (numpy), one head of one sequence at a time, and
bounds of what an evaluation in fp32 (with the roundings to a 16-bit type that the interface allows) may be off.

The bounds are first-order rounding-error sums, u = 2^-24, h = half a step of the type the products' operands and the outputs are
rounded to (bf16 2^-8; fp32: operands are not rounded, h_op = 0, outputs u):
  score   a product of d terms, a factor, a sum, a change of base: (d + 8) u (scale sum |q||k| + |bias|) =: e_s
  p       2 e_s (numerator and denominator) + the chain of the row sum and of the exponential (n_k + 32) u
  out     sum p |v| (e_p + h_op) + h |out|;   lse: e_s + (n_k + 32) u + u |lse|
  ds      e_p |ds| + p (d + 8) u (sum |do||v| + sum |do||o|), and h_op |ds| as an operand
  dq, dk, dv: the errors of their operands times the other operand's size, the chain of the sum, and h of the result
  dtable  the errors of ds and the chain of its sum
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24
HIDDEN = -1e30


def bucket_of(rel: int, buckets: int, max_distance: int, bidirectional: bool) -> int:
    """In whole numbers: bucket e + k begins at the smallest r with (r / e)^m >= (max_distance / e)^k."""
    n = buckets // 2 if bidirectional else buckets
    r, first = (abs(rel), n if rel > 0 else 0) if bidirectional else (max(0, -rel), 0)
    e = n // 2
    m = n - e
    if r < e:
        return first + r
    r, k = min(r, max_distance), 0
    while k + 1 < m and r ** m * e ** (k + 1) >= max_distance ** (k + 1) * e ** m:
        k += 1
    return first + e + k


def bucket_grid(nq: int, nk: int, shift: int, buckets: int, max_distance: int, bidirectional: bool) -> np.ndarray:
    by = {r: bucket_of(r, buckets, max_distance, bidirectional) for r in range(-nq - shift, nk - shift + 1)}
    return np.array([[by[j - i - shift] for j in range(nk)] for i in range(nq)], dtype=np.int64).reshape(nq, nk)


def position_bias(table, nq, nk, offset, max_distance, bidirectional):
    grid = bucket_grid(nq, nk, offset, table.shape[0], max_distance, bidirectional)
    return np.moveaxis(table[grid], 2, 0)


def position_bias_backward(dbias, buckets, offset, max_distance, bidirectional):
    """dbias [b, h, q, k] -> (dtable [buckets, h], sum of |dbias| by bucket)."""
    b, h, nq, nk = dbias.shape
    grid = bucket_grid(nq, nk, offset, buckets, max_distance, bidirectional).reshape(-1)
    out, size = np.zeros((buckets, h)), np.zeros((buckets, h))
    for k in range(h):
        out[:, k] = np.bincount(grid, weights=dbias[:, k].sum(0).reshape(-1), minlength=buckets)
        size[:, k] = np.bincount(grid, weights=np.abs(dbias[:, k]).sum(0).reshape(-1), minlength=buckets)
    return out, size


def attention(q, k, v, scale, causal=False, q_lens=None, k_lens=None, bias=None, dout=None, saved=None, half_step=U, operand_step=0.0):
    """q [b, i, h, d], k / v [b, j, g, d] -> dict of results and, under the same names in "bound", how far an fp32 evaluation may
    be off.  bias = (table [buckets, heads], max_distance, bidirectional).  With dout also the gradients, from the output and
    lse of `saved` (what the evaluation under test was given)."""
    B, NQ, H, D = q.shape
    NK, G = k.shape[1], k.shape[2]
    with np.errstate(all="ignore"):
        return _attention(q, k, v, scale, causal, q_lens, k_lens, bias, dout, saved, half_step, operand_step, B, NQ, H, D, NK, G)


def _attention(q, k, v, scale, causal, q_lens, k_lens, bias, dout, saved, half_step, operand_step, B, NQ, H, D, NK, G):
    z = lambda *s: np.zeros(s)  # noqa: E731
    r = dict(out=z(B, NQ, H, D), lse=np.full((B, H, NQ), -np.inf))
    e = dict(out=z(B, NQ, H, D), lse=z(B, H, NQ))
    if dout is not None:
        for n, s in (("dq", q), ("dk", k), ("dv", v)):
            r[n], e[n] = z(*s.shape), z(*s.shape)
        if bias is not None:
            r["dtable"], e["dtable"], size_t = z(*bias[0].shape), z(*bias[0].shape), z(*bias[0].shape)
    chain_k, chain_q = (NK + 32) * U, (NQ * (H // G) + 32) * U
    sums = dict(dk=z(*k.shape), dv=z(*v.shape))
    for b in range(B):
        nq = NQ if q_lens is None else int(np.clip(q_lens[b], 0, NQ))
        nk = NK if k_lens is None else int(np.clip(k_lens[b], 0, NK))
        if nq == 0 or nk == 0:
            continue
        shift = nk - nq if causal else 0
        seen = np.ones((nq, nk), bool)
        if causal:
            seen = np.arange(nk)[None, :] <= np.arange(nq)[:, None] + shift
        grid = None if bias is None else bucket_grid(nq, nk, shift, bias[0].shape[0], bias[1], bias[2])
        for h in range(H):
            g = h // (H // G)
            qq, kk, vv = q[b, :nq, h], k[b, :nk, g], v[b, :nk, g]
            s, size = scale * (qq @ kk.T), abs(scale) * (np.abs(qq) @ np.abs(kk).T)
            ok = seen
            if grid is not None:
                t = bias[0][:, h][grid]
                ok = seen & (t > HIDDEN)
                s, size = s + np.where(ok, t, 0.0), size + np.where(ok, np.abs(t), 0.0)
            s = np.where(ok, s, -np.inf)
            some = ok.any(1)
            top = np.where(some, s.max(1), 0.0)
            w = np.exp(s - top[:, None])
            total = np.where(some, w.sum(1), 1.0)
            e_s = (D + 8) * U * np.where(ok, size, 0.0).max(1)
            lse = np.where(some, top + np.log(total), -np.inf)
            r["lse"][b, h, :nq] = lse
            e["lse"][b, h, :nq] = np.where(some, e_s + chain_k + U * np.abs(lse), 0.0)
            p = w / total[:, None]
            o = p @ vv
            e_p = 2 * e_s[:, None] + chain_k
            r["out"][b, :nq, h] = o
            e["out"][b, :nq, h] = (p * (e_p + operand_step + chain_k)) @ np.abs(vv) + half_step * np.abs(o)
            if dout is None:
                continue
            do, oo, ls = dout[b, :nq, h], saved[0][b, :nq, h], saved[1][b, h, :nq]
            p = np.where(ok & np.isfinite(ls)[:, None], np.exp(np.where(ok, s, 0.0) - np.where(np.isfinite(ls), ls, 0.0)[:, None]), 0.0)
            ds = p * (do @ vv.T - (do * oo).sum(1, keepdims=True))
            e_p = e_s[:, None] + (32 + 2 * np.abs(np.where(np.isfinite(ls), ls, 0.0)))[:, None] * U
            e_ds = e_p * np.abs(ds) + p * (D + 8) * U * (np.abs(do) @ np.abs(vv).T + (np.abs(do) * np.abs(oo)).sum(1, keepdims=True))
            e_op = e_ds + operand_step * np.abs(ds)
            r["dq"][b, :nq, h] = scale * (ds @ kk)
            e["dq"][b, :nq, h] = abs(scale) * ((e_op + chain_k * np.abs(ds)) @ np.abs(kk)) + half_step * np.abs(r["dq"][b, :nq, h])
            r["dk"][b, :nk, g] += scale * (ds.T @ qq)
            sums["dk"][b, :nk, g] += abs(scale) * ((e_op + chain_q * np.abs(ds)).T @ np.abs(qq))
            r["dv"][b, :nk, g] += p.T @ do
            sums["dv"][b, :nk, g] += (p * (e_p + operand_step + chain_q)).T @ np.abs(do)
            if grid is not None:
                n = bias[0].shape[0]
                r["dtable"][:, h] += np.bincount(grid.reshape(-1), weights=ds.reshape(-1), minlength=n)
                e["dtable"][:, h] += np.bincount(grid.reshape(-1), weights=(e_ds + (NQ + NK + 64) * U * np.abs(ds)).reshape(-1), minlength=n)
    if dout is not None:
        for n in ("dk", "dv"):
            e[n] = sums[n] + half_step * np.abs(r[n])
        if bias is not None:
            e["dtable"] += U * np.abs(r["dtable"])
    r["bound"] = e
    return r
