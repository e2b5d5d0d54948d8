"""The measured work of the operators of the training model's Transformer layers:
attention, its backward pass, and the learned relative position bias.

Four kinds of case, told apart by case["op"]:

  forward    attention of a batch: the output and the log-sum-exp of every row.
  backward   its gradient: dq, dk, dv and the gradient of the position table,
             from q, k, v, the saved output and log-sum-exp, and dout.
  bias       the position bias as a tensor of [heads, queries, keys].
  bias_grad  the gradient of its table from the gradient of that tensor, which
             is summed over the batch.

Lengths of a padded batch are a function of the case: they fall from the full
length to about half of it over the batch ("ragged"), and the last sequence is
empty where "empty" says so.  Tensors are [batch, token, head, feature]; with
"packed" the queries, keys and values of a self-attention are slices of one
[batch, token, 3, heads, feature] tensor (keys and values of one, where the
lengths or head counts differ), as a fused projection leaves them.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------

def _attention(op, dtype, batch, q_len, k_len, heads, kv_heads, dim, causal=False, buckets=0, max_distance=0,
               bidirectional=True, ragged=False, empty=False, packed=False):
    return dict(op=op, dtype=dtype, batch=batch, q_len=q_len, k_len=k_len, heads=heads, kv_heads=kv_heads, dim=dim,
                causal=causal, buckets=buckets, max_distance=max_distance, bidirectional=bidirectional, ragged=ragged,
                empty=empty, packed=packed)


def _bias(op, dtype, batch, heads, q_len, k_len, offset=0, buckets=32, max_distance=128, bidirectional=True):
    return dict(op=op, dtype=dtype, batch=batch, heads=heads, q_len=q_len, k_len=k_len, offset=offset, buckets=buckets,
                max_distance=max_distance, bidirectional=bidirectional)


def listed():
    return [
        # A small fp32 layer on short sentences: the smallest call, where latency is all of it.
        dict(_attention("forward", "f32", 4, 32, 32, 2, 2, 64, ragged=True), name="short_forward"),
        # One encoder layer of a mixed-precision training step on a padded batch, with a position bias.
        dict(_attention("forward", "bf16", 32, 128, 128, 12, 12, 64, buckets=32, max_distance=128, ragged=True, packed=True),
             name="encoder_forward"),
        # A long causal document with shared key heads: all arithmetic.
        dict(_attention("forward", "bf16", 2, 8192, 8192, 16, 4, 128, causal=True), name="long_forward"),
        # The next token of sixteen sequences of different lengths against their keys: the keys are read once.
        dict(_attention("forward", "bf16", 16, 1, 8192, 32, 8, 128, causal=True, buckets=32, max_distance=128,
                        bidirectional=False, ragged=True), name="one_token_forward"),
        # Backward of an encoder layer at the size of the full stack, padded batch, position table trained.
        dict(_attention("backward", "bf16", 64, 256, 256, 12, 12, 64, buckets=32, max_distance=128, ragged=True, packed=True),
             name="encoder_backward"),
        # Backward of a long causal layer with shared key heads.
        dict(_attention("backward", "bf16", 2, 4096, 4096, 16, 4, 128, causal=True), name="long_backward"),
        # fp32 training at an odd sequence length.
        dict(_attention("backward", "f32", 24, 197, 197, 12, 12, 64), name="fp32_backward"),
        # A decoder's attention to the encoder's output: lengths that differ, a small odd head, an empty sequence.
        dict(_attention("backward", "bf16", 6, 77, 331, 6, 6, 40, buckets=20, max_distance=50, ragged=True, empty=True,
                        packed=True), name="cross_backward"),
        # The bias of a short sentence as a tensor.
        dict(_bias("bias", "f32", 1, 8, 77, 77), name="short_bias"),
        # The bias of a long document in the type of mixed precision.
        dict(_bias("bias", "bf16", 1, 16, 4096, 4096, bidirectional=False), name="long_bias"),
        # Gradient of the table from the score gradients of a batch.
        dict(_bias("bias_grad", "bf16", 16, 12, 256, 256), name="batch_bias_gradient"),
        # The same from one long odd-sized score gradient in fp32.
        dict(_bias("bias_grad", "f32", 2, 16, 2047, 2111, offset=64), name="long_bias_gradient"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_buckets(rng, bidirectional):
    buckets = 2 * rng.choice((16, 16, 8, _log(rng, 2, 40)))
    side = buckets // 2 if bidirectional else buckets
    return buckets, max(side, rng.choice((128, 128, 64, _log(rng, 16, 1024))))


def _draw_attention(rng, op):
    dtype = rng.choice(("bf16", "bf16", "f32"))
    dim = rng.choice((64, 64, 128, 128, 32, 80, 96, 8 * rng.randint(2, 16), rng.randint(8, 128)))
    kv_heads = rng.choice((1, 2, 4, 8, 12, rng.randint(1, 12)))
    heads = kv_heads * rng.choice((1, 1, 2, 4) if kv_heads <= 8 else (1,))
    causal = rng.random() < 0.5
    if op == "forward" and rng.random() < 0.3:
        q_len = rng.choice((1, 1, 1, rng.randint(2, 24)))
        k_len = max(q_len, _log(rng, 64, 16384))
    else:
        q_len = _log(rng, 16, 4096)
        k_len = q_len if rng.random() < 0.7 else _log(rng, 16, 4096)
    # no more pairs times features than the long listed case of the kind, an eighth of them in fp32
    most = {"forward": 1.0e11, "backward": 2.5e10}[op] / (1 if dtype == "bf16" else 8)
    batch = _log(rng, 1, 64)
    while batch * heads * q_len * k_len > min(5e8, most / dim) or batch * kv_heads * k_len * dim > 2 ** 27:
        if batch > 1:
            batch = (batch + 1) // 2
        else:
            q_len, k_len = (q_len + 1) // 2, (k_len + 1) // 2
    buckets, max_distance, bidirectional = 0, 0, True
    if rng.random() < 0.5:
        bidirectional = not causal or rng.random() < 0.3
        buckets, max_distance = _draw_buckets(rng, bidirectional)
    ragged = rng.random() < 0.5
    return _attention(op, dtype, batch, q_len, k_len, heads, kv_heads, dim, causal, buckets, max_distance, bidirectional,
                      ragged, ragged and rng.random() < 0.3, rng.random() < 0.5)


def draw(rng):
    op = rng.choice(("forward", "forward", "backward", "backward", "backward", "bias", "bias_grad"))
    if op in ("forward", "backward"):
        return _draw_attention(rng, op)
    dtype = rng.choice(("bf16", "f32"))
    bidirectional = rng.random() < 0.6
    buckets, max_distance = _draw_buckets(rng, bidirectional)
    heads = rng.choice((4, 8, 12, 16, rng.randint(1, 24)))
    q_len = _log(rng, 16, 4096)
    k_len = q_len if rng.random() < 0.5 else _log(rng, 16, 4096)
    batch = 1 if op == "bias" else _log(rng, 1, 32)
    while batch * heads * q_len * k_len > 1.3e8:
        if batch > 1:
            batch = (batch + 1) // 2
        else:
            q_len, k_len = (q_len + 1) // 2, (k_len + 1) // 2
    offset = rng.choice((0, 0, max(0, k_len - q_len), rng.randint(0, k_len)))
    return _bias(op, dtype, batch, heads, q_len, k_len, offset, buckets, max_distance, bidirectional)


# ---- what a program has in hand before the call --------------------------------------------------

def _lengths(case):
    """Lengths of the sequences of a case, (queries, keys), or None for a batch without padding."""
    if not case["ragged"]:
        return None, None
    def of(n):
        out = [max(1, n - i * n // (2 * case["batch"])) for i in range(case["batch"])]
        if case["empty"] and case["batch"] > 1:
            out[-1] = 0
        return out
    if case["q_len"] == case["k_len"]:
        return of(case["q_len"]), of(case["k_len"])       # self-attention: the same tokens
    return None, of(case["k_len"])


def _randn(g, *shape, dtype=torch.float32, gain=1.0):
    return (torch.randn(shape, generator=g, device=DEVICE) * gain).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]
    s = dict(case=dict(case))
    if case["buckets"]:
        s["table"] = _randn(g, case["buckets"], case["heads"], gain=0.7)
    if case["op"] == "bias":
        return s
    if case["op"] == "bias_grad":
        s["dbias"] = _randn(g, case["batch"], case["heads"], case["q_len"], case["k_len"], dtype=t, gain=0.01)
        return s
    b, nq, nk, h, hk, d = (case[k] for k in ("batch", "q_len", "k_len", "heads", "kv_heads", "dim"))
    if case["packed"] and nq == nk and h == hk:
        s["q"], s["k"], s["v"] = _randn(g, b, nq, 3, h, d, dtype=t).unbind(2)
    else:
        s["q"] = _randn(g, b, nq, h, d, dtype=t)
        if case["packed"]:
            s["k"], s["v"] = _randn(g, b, nk, 2, hk, d, dtype=t).unbind(2)
        else:
            s["k"], s["v"] = _randn(g, b, nk, hk, d, dtype=t), _randn(g, b, nk, hk, d, dtype=t)
    ql, kl = _lengths(case)
    s["q_lens"] = None if ql is None else torch.tensor(ql, dtype=torch.int32, device=DEVICE)
    s["k_lens"] = None if kl is None else torch.tensor(kl, dtype=torch.int32, device=DEVICE)
    if case["op"] == "backward":                         # what the forward pass saved, and the gradient that arrives
        s["out"], s["lse"] = _plain_forward(s)
        s["dout"] = _randn(g, b, nq, h, d, dtype=t, gain=0.1)
    return s


# ---- plain forms --------------------------------------------------------------------------------

def _bucket_lut(case, device):
    """Bucket of every distance key - query in [-M, M]; farther ones have the bucket of the nearest end."""
    n = case["buckets"] // 2 if case["bidirectional"] else case["buckets"]
    exact_ones = n // 2
    wide, far = n - exact_ones, case["max_distance"]
    at = [exact_ones * (far / exact_ones) ** (k / wide) for k in range(1, wide)]
    at = [round(x) if abs(x - round(x)) <= 1e-12 * x else x for x in at]
    borders = torch.tensor([float(i) for i in range(1, exact_ones + 1)] + at, dtype=torch.float64, device=device)
    rel = torch.arange(-far, far + 1, device=device)
    dist = rel.abs() if case["bidirectional"] else (-rel).clamp(min=0)
    bucket = (dist[:, None] >= borders).sum(1)
    return bucket + n * (rel > 0) if case["bidirectional"] else bucket


def _plain_bias(case, table, rel):
    """table entries [..., heads] of the distances rel = key position - query position."""
    far = case["max_distance"]
    return table[_bucket_lut(case, table.device)[rel.clamp(-far, far) + far]]


def _plain_scores(s):
    """fp32 scores [b, heads, q, k], minus infinity where a pair is hidden, and the distances and mask."""
    case, q, k = s["case"], s["q"], s["k"]
    b, nq, h, d = q.shape
    nk, hk = k.shape[1], k.shape[2]
    scores = torch.matmul((q.float() * (1.0 / math.sqrt(d))).reshape(b, nq, hk, h // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d),
                          k.float().permute(0, 2, 3, 1).contiguous()).reshape(b, h, nq, nk)
    full = lambda n: torch.full((b,), n, dtype=torch.int32, device=q.device)  # noqa: E731
    ql = full(nq) if s["q_lens"] is None else s["q_lens"]
    kl = full(nk) if s["k_lens"] is None else s["k_lens"]
    i, j = torch.arange(nq, device=q.device)[:, None], torch.arange(nk, device=q.device)[None, :]
    rel = (j - i)[None]
    seen = (i < ql[:, None, None]) & (j < kl[:, None, None])
    if case["causal"]:
        rel = rel - (kl - ql)[:, None, None]
        seen = seen & (rel <= 0)
    if case["buckets"]:
        scores += _plain_bias(case, s["table"], rel).permute(0, 3, 1, 2)
    scores.masked_fill_(~seen[:, None], float("-inf"))
    return scores, rel


def _shared(x, hk):
    """[b, heads, q, k] -> [b, key heads, heads of the group * q, k]"""
    return x.reshape(x.shape[0], hk, -1, x.shape[-1])


def _plain_forward(s):
    q, k, v = s["q"], s["k"], s["v"]
    b, nq, h, d = q.shape
    scores, _ = _plain_scores(s)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = (scores - top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p /= total.clamp(min=1e-30)
    out = torch.matmul(_shared(p, k.shape[2]), v.float().transpose(1, 2).contiguous()).reshape(b, h, nq, d)
    return out.transpose(1, 2).to(q.dtype).contiguous(), lse


def _plain_backward(s):
    case, q, k, v = s["case"], s["q"], s["k"], s["v"]
    b, nq, h, d = q.shape
    nk, hk = k.shape[1], k.shape[2]
    scores, rel = _plain_scores(s)
    p = (scores - s["lse"].clamp(min=-1e30)[..., None]).exp_()
    dout = s["dout"].float().transpose(1, 2)
    delta = (dout * s["out"].float().transpose(1, 2)).sum(-1, keepdim=True)
    dout = _shared(dout, hk)
    dv = torch.matmul(_shared(p, hk).transpose(2, 3), dout)
    ds = torch.matmul(dout, v.float().permute(0, 2, 3, 1).contiguous()).reshape(b, h, nq, nk)
    ds = (ds - delta).mul_(p)
    scale = 1.0 / math.sqrt(d)
    dq = torch.matmul(_shared(ds, hk), k.float().transpose(1, 2).contiguous()).reshape(b, h, nq, d) * scale
    dk = torch.matmul(_shared(ds, hk).transpose(2, 3), _shared(q.float().transpose(1, 2), hk)) * scale
    grads = {"dq": dq.transpose(1, 2).to(q.dtype), "dk": dk.transpose(1, 2).to(q.dtype), "dv": dv.transpose(1, 2).to(q.dtype)}
    if case["buckets"]:
        if rel.shape[0] == 1:                             # the same distances in every sequence
            ds = ds.sum(0, keepdim=True, dtype=torch.float64)
        grads["dtable"] = _plain_table_grad(case, ds, rel[:, 0, 0])
    return grads


def _plain_table_grad(case, ds, first):
    """Sum of ds [b, heads, q, k] by bucket, in 64 bits -> [buckets, heads]; first [b]: distance of the first key from the first query."""
    b, h, nq, nk = ds.shape
    rows = torch.nn.functional.pad(ds.flip(2), (0, nq)).reshape(b, h, -1)[..., :-nq].reshape(b, h, nq, nq + nk - 1)
    by_distance = rows.sum(2, dtype=torch.float64)        # row q moved so that distances lie below each other
    far = case["max_distance"]
    rel = first[:, None] - (nq - 1) + torch.arange(nq + nk - 1, device=ds.device)
    which = _bucket_lut(case, ds.device)[rel.clamp(-far, far) + far]
    one = (which[..., None] == torch.arange(case["buckets"], device=ds.device)).double()
    return torch.matmul(by_distance, one).sum(0).t().float().contiguous()


def _distances(case):
    return torch.arange(case["k_len"], device=DEVICE)[None, :] - torch.arange(case["q_len"], device=DEVICE)[:, None] - case["offset"]


def _plain(s):
    case = s["case"]
    if case["op"] == "forward":
        out, lse = _plain_forward(s)
        return {"out": out, "lse": lse}
    if case["op"] == "backward":
        return _plain_backward(s)
    if case["op"] == "bias":
        return _plain_bias(case, s["table"], _distances(case)).to(TYPES[case["dtype"]]).permute(2, 0, 1).contiguous()
    first = torch.tensor([-case["offset"]], device=DEVICE)
    return _plain_table_grad(case, s["dbias"].sum(0, keepdim=True, dtype=torch.float64), first)


# ---- one pass -------------------------------------------------------------------------------------

def run(state):
    if own:
        from paper_2201_06227_amd import binding as eg
        case = state["case"]
        op = case["op"]
        bias = eg.PositionBias(state["table"], case["max_distance"], case["bidirectional"]) if case["buckets"] else None
        if op == "bias":
            return eg.position_bias(bias, case["q_len"], case["k_len"], offset=case["offset"], dtype=TYPES[case["dtype"]])
        if op == "bias_grad":
            return eg.position_bias_backward(state["dbias"], bias, offset=case["offset"])
        how = dict(causal=case["causal"], bias=bias, q_lens=state["q_lens"], k_lens=state["k_lens"])
        if op == "forward":
            out, lse = eg.attention(state["q"], state["k"], state["v"], **how)
            return {"out": out, "lse": lse}
        dq, dk, dv, dtable = eg.attention_backward(state["dout"], state["q"], state["k"], state["v"], state["out"], state["lse"], **how)
        return {"dq": dq, "dk": dk, "dv": dv, **({"dtable": dtable} if bias else {})}
    return _plain(state)


# ---- cost and definition ----------------------------------------------------------------------------

def _pairs(case):
    """Visible pairs of one head, summed over the batch."""
    ql, kl = _lengths(case)
    total = 0
    for i in range(case["batch"]):
        n, m = case["q_len"] if ql is None else ql[i], case["k_len"] if kl is None else kl[i]
        if not case["causal"]:
            total += n * m
        else:                                             # query r sees m - n + r + 1 keys, where that is positive
            hidden = max(0, n - m)
            rows = n - hidden
            total += rows * (m - n + hidden + 1) + rows * (rows - 1) // 2
    return total


def work(case):
    size = {"bf16": 2, "f32": 4}[case["dtype"]]
    if case["op"] in ("bias", "bias_grad"):
        cells = case["batch"] * case["heads"] * case["q_len"] * case["k_len"]
        return {"bytes": cells * size + 4 * case["buckets"] * case["heads"], "flops": cells if case["op"] == "bias_grad" else 0}
    ql, kl = _lengths(case)
    tokens_q = case["batch"] * case["q_len"]
    tokens_k = case["batch"] * case["k_len"] if kl is None else sum(kl)
    rows = tokens_q * case["heads"] * case["dim"] * size
    keys = tokens_k * case["kv_heads"] * case["dim"] * size
    stats = 4 * tokens_q * case["heads"] + 4 * case["buckets"] * case["heads"]
    if case["op"] == "forward":
        return {"bytes": 2 * rows + 2 * keys + stats, "flops": 4 * _pairs(case) * case["heads"] * case["dim"]}
    return {"bytes": 4 * rows + 4 * keys + stats, "flops": 10 * _pairs(case) * case["heads"] * case["dim"]}


def _bucket_of(distance, n, far):
    """Whole numbers alone: the border of bucket e + k is the smallest r with (r / e)^m >= (far / e)^k."""
    e = n // 2
    m = n - e
    if distance < e:
        return distance
    k = 0
    while k + 1 < m and distance ** m * e ** (k + 1) >= far ** (k + 1) * e ** m:
        k += 1
    return e + k


def _exact_buckets(case, first, count):
    """Buckets of the distances first, first + 1, ... (key position - query position)."""
    n = case["buckets"] // 2 if case["bidirectional"] else case["buckets"]
    near = [_bucket_of(r, n, case["max_distance"]) for r in range(case["max_distance"] + 1)]
    got = []
    for rel in range(first, first + count):
        r = abs(rel) if case["bidirectional"] else max(0, -rel)
        got.append(near[min(r, case["max_distance"])] + (n if case["bidirectional"] and rel > 0 else 0))
    return torch.tensor(got, device=DEVICE)


def _toeplitz(values, nq, nk):
    """[q, k] tensor of values[(k - q) + q_len - 1]."""
    return values.unfold(0, nk, 1).flip(0)


def exact(case, seed):
    s = prepare(case, seed)
    nq, nk = case["q_len"], case["k_len"]
    if case["op"] in ("bias", "bias_grad"):
        which = _exact_buckets(case, -case["offset"] - nq + 1, nq + nk - 1)
        if case["op"] == "bias":
            return torch.stack([_toeplitz(s["table"][:, h].double()[which], nq, nk) for h in range(case["heads"])])
        grad = torch.zeros(case["buckets"], case["heads"], dtype=torch.float64, device=DEVICE)
        grid = _toeplitz(which, nq, nk).reshape(-1)
        for h in range(case["heads"]):
            total = sum(s["dbias"][b, h].double() for b in range(case["batch"]))
            grad[:, h] = torch.bincount(grid, weights=total.reshape(-1), minlength=case["buckets"])
        return grad
    group = case["heads"] // case["kv_heads"]
    ql, kl = _lengths(case)
    like = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=DEVICE)  # noqa: E731
    out, lse = like(s["q"]), torch.full((case["batch"], case["heads"], nq), -math.inf, dtype=torch.float64, device=DEVICE)
    dq, dk, dv = like(s["q"]), like(s["k"]), like(s["v"])
    dtable = torch.zeros(case["buckets"], case["heads"], dtype=torch.float64, device=DEVICE)
    for b in range(case["batch"]):
        n, m = nq if ql is None else ql[b], nk if kl is None else kl[b]
        if n == 0 or m == 0:
            continue
        shift = m - n if case["causal"] else 0
        which = _toeplitz(_exact_buckets(case, -shift - n + 1, n + m - 1), n, m) if case["buckets"] else None
        blind = torch.ones(n, m, dtype=torch.bool, device=DEVICE).triu(shift + 1) if case["causal"] else None
        for h in range(case["heads"]):
            q, k, v = s["q"][b, :n, h].double(), s["k"][b, :m, h // group].double(), s["v"][b, :m, h // group].double()
            x = q @ k.t() / math.sqrt(case["dim"])
            if which is not None:
                x += s["table"][:, h].double()[which]
            if blind is not None:
                x[blind] = -math.inf
            if case["op"] == "forward":
                lse[b, h, :n] = torch.logsumexp(x, 1)
                out[b, :n, h] = torch.softmax(x, 1).nan_to_num(0.0) @ v
                continue
            p = torch.exp(x - s["lse"][b, h, :n, None].double()).nan_to_num(0.0)
            do = s["dout"][b, :n, h].double()
            ds = p * (do @ v.t() - (do * s["out"][b, :n, h].double()).sum(1, keepdim=True))
            dq[b, :n, h] = ds @ k / math.sqrt(case["dim"])
            dk[b, :m, h // group] += ds.t() @ q / math.sqrt(case["dim"])
            dv[b, :m, h // group] += p.t() @ do
            if which is not None:
                dtable[:, h] += torch.bincount(which.reshape(-1), weights=ds.reshape(-1), minlength=case["buckets"])
    if case["op"] == "forward":
        return {"out": out, "lse": lse}
    return {"dq": dq, "dk": dk, "dv": dv, **({"dtable": dtable} if case["buckets"] else {})}
