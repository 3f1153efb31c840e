"""The measured cases of the sequence operators: layer norm, and attention over packed sequences with a learned bias by distance.

  op        layer_norm | layer_norm_backward | attention | attention_backward
layer norm
  rows, cols; io: type of the rows; params: type of weight and bias (f32 | f16 | bf16)
attention
  N         sequences, packed one after the other
  lengths   keys of a sequence: "fixed L" | "uniform lo hi" | "lognormal mu sigma cap" (the lengths' spread is the case's, their order the seed's)
  queries   "all": every token is a query and a key, q, k and v are column blocks of one matrix; "last M": the last M tokens of a
            sequence (fewer where it is shorter) attend to its whole cache; M = 1 is a decoding step
  room      share of the cache's rows that no token has filled yet ("last" only)
  heads, kv_heads, dim; causal; io: type of q, k, v, out and the gradients (the bias table has it too); ids: type of offsets and lengths
  buckets   0: no bias; otherwise the table's buckets per head, distances beyond `far` in the last one
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
_IO = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_IDX = {"i64": torch.int64, "i32": torch.int32}
_BYTES = {"i64": 8, "i32": 4, "f32": 4, "f16": 2, "bf16": 2}


def _norm(name, op, rows, cols, io, params):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "io": io, "params": params}


def _attend(name, op, N, lengths, heads, kv_heads, dim, io, queries="all", room=0.0, causal=True, buckets=32, far=128, ids="i64"):
    return {"name": name, "op": op, "N": N, "lengths": lengths, "queries": queries, "room": room, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "causal": causal, "io": io, "ids": ids, "buckets": buckets, "far": far}


def listed():
    return [
        # the newest event of each sample of a serving request: latency only
        _norm("norm_request", "layer_norm", 32, 192, "f32", "f32"),
        # the events of a large batch, rows as the lookup leaves them
        _norm("norm_events", "layer_norm", 1_000_003, 128, "bf16", "f32"),
        # the same rows in training, at a middle width
        _norm("norm_events_backward", "layer_norm_backward", 262_147, 256, "bf16", "f32"),
        # wide rows of an odd width in full precision: few rows, the weights' gradient counts
        _norm("norm_wide_backward", "layer_norm_backward", 8_001, 1_021, "f32", "f32"),
        # one new event for each of a request's users against their short histories
        _attend("request_step", "attention", 32, "lognormal 2 1 500", 4, 4, 32, "f32", queries="last 1", ids="i32"),
        # one new event against very long histories, many heads on few keys, caches with room left
        _attend("long_cache_step", "attention", 24, "uniform 2000 65536", 16, 2, 128, "bf16", queries="last 1", room=0.2, buckets=0),
        # a training batch of event sequences: long-tailed lengths, most of them short
        _attend("events_forward", "attention", 4096, "lognormal 2 1 500", 4, 4, 32, "bf16"),
        # whole long sequences, grouped heads
        _attend("long_forward", "attention", 2, "uniform 4000 8000", 16, 4, 128, "bf16", buckets=0),
        # a few dozen new events behind a middling history
        _attend("append_forward", "attention", 48, "uniform 100 4000", 8, 8, 64, "f16", queries="last 61", room=0.1, ids="i32"),
        # the gradients of the training batch, the bias table's among them
        _attend("events_backward", "attention_backward", 4096, "lognormal 2 1 500", 4, 4, 32, "bf16"),
        # ... of long sequences with grouped heads
        _attend("long_backward", "attention_backward", 4, "uniform 1000 4096", 8, 2, 64, "f16"),
        # ... in full precision, every event seeing all others
        _attend("full_precision_backward", "attention_backward", 64, "uniform 1 200", 2, 2, 64, "f32", causal=False, ids="i32"),
    ]


def draw(rng):
    def spread(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    op = rng.choice(("layer_norm", "layer_norm_backward", "attention", "attention", "attention", "attention_backward", "attention_backward"))
    io = rng.choice(("f32", "f16", "bf16", "bf16"))
    if op.startswith("layer_norm"):
        cols = rng.choice((int(spread(8, 2048)), 8 * int(spread(1, 256))))
        rows = int(spread(1, 1.2e8 / cols if op == "layer_norm" else 6.0e7 / cols))
        case = _norm("", op, rows, cols, io, rng.choice(("f32", "f32", io)))
    else:
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
        dim = rng.choice((16, 32, 32, 64, 64, 80, 96, 128, 128))
        queries = "all" if op == "attention_backward" else rng.choice(("all", "all", "last 1", "last 1", "last %d" % int(spread(2, 200))))
        one = queries == "last 1"
        longest = spread(20, 60_000 if one else 6_000)
        shape = rng.choice(("fixed %d" % longest, "uniform %d %d" % (longest / spread(1, 30), longest), "lognormal %.2f 1 %d" % (math.log(longest / 12 + 1), longest)))
        N = max(1, int(spread(1, 4000)))
        most = int(shape.split()[-1])
        asking = most if queries == "all" else min(most, int(queries.split()[1]))
        # pairs of a padded batch, their operations, and the tokens
        limit = 4.0e8 if op == "attention_backward" else 1.0e9
        while N > 1 and (N * heads * most * asking > limit or N * heads * most * asking * dim > 64 * limit or N * most * kv_heads * dim > 2.0e8):
            N = N * 2 // 3
        while heads > kv_heads and heads * most * asking > limit:
            heads -= kv_heads
        case = _attend("", op, N, shape, heads, kv_heads, dim, io, queries, 0.0 if queries == "all" else rng.choice((0.0, 0.15)), rng.random() < 0.8,
                       rng.choice((0, 16, 32, 48)), rng.choice((32, 128, 500)), rng.choice(("i64", "i32")))
    del case["name"]
    return case


def _lengths(case):
    """Keys and queries of every sequence, in an order of no meaning."""
    at = (0.5 + np.arange(case["N"]) * 0.6180339887498949) % 1.0
    kind, *p = case["lengths"].split()
    p = [float(x) for x in p]
    if kind == "fixed":
        n = np.full(case["N"], p[0])
    elif kind == "uniform":
        n = p[0] + at * (p[1] - p[0])
    else:
        z = torch.special.ndtri(torch.from_numpy(np.clip(at, 1e-6, 1 - 1e-6))).numpy()
        n = np.exp(p[0] + p[1] * z).clip(1, p[2])
    n = n.round().astype(np.int64).clip(1)
    return n, (n if case["queries"] == "all" else np.minimum(n, int(case["queries"].split()[1])))


def work(case):
    w = _BYTES[case["io"]]
    if case["op"].startswith("layer_norm"):
        n, p = case["rows"] * case["cols"], case["cols"] * _BYTES[case["params"]]
        if case["op"] == "layer_norm":
            return {"bytes": 2 * n * w + 2 * p + 8 * case["rows"], "flops": 8 * n}
        return {"bytes": 3 * n * w + 3 * p + 8 * case["rows"], "flops": 14 * n}
    nk, nq = _lengths(case)
    pairs = int((nq * nk - (nq * (nq - 1) // 2 if case["causal"] else 0)).sum()) * case["heads"]
    q, k = int(nq.sum()) * case["heads"] * case["dim"], int(nk.sum()) * case["kv_heads"] * case["dim"]
    table = case["heads"] * case["buckets"] * w
    if case["op"] == "attention":
        return {"bytes": (2 * q + 2 * k) * w + table, "flops": 4 * case["dim"] * pairs}
    return {"bytes": (4 * q + 4 * k) * w + 4 * int(nq.sum()) * case["heads"] + 2 * table, "flops": 10 * case["dim"] * pairs}


def _bucket_map(case):
    """The bucket of every distance -far .. far: the nearest distances one each, the further ones by their logarithm; distances
    ahead of the query, which only a batch without causal order has, share the other half of the buckets."""
    far, n = case["far"], case["buckets"]
    d = np.arange(-far, far + 1)
    half = n if case["causal"] else n // 2
    near = half // 2
    a = np.abs(d)
    log = near + (np.log(np.maximum(a, 1) / max(near, 1)) / math.log(max(far, near + 1) / max(near, 1)) * (half - 1 - near)).astype(np.int64)
    b = np.where(a < near, a, np.clip(log, 0, half - 1))
    if not case["causal"]:
        b = b + half * (d < 0)
    return torch.from_numpy(b.astype(np.int32)).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    io = _IO[case["io"]]

    def normal(*shape, mul=1.0, add=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(mul).add_(add)

    s = {"case": case}
    if own:
        from paper_2508_03854_amd import TBE
        s["tbe"] = TBE([16], [8])
    if case["op"].startswith("layer_norm"):
        rows, cols, params = case["rows"], case["cols"], _IO[case["params"]]
        s |= {"x": normal(rows, cols, mul=0.7, add=0.2).to(io), "weight": normal(cols, mul=0.2, add=1.0).to(params), "bias": normal(cols, mul=0.2).to(params)}
        if case["op"] == "layer_norm_backward":
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square_().mean(1) + EPS)
            s["grad"] = normal(rows, cols).to(io)
            if own:
                s["workspace"] = s["tbe"].alloc_layer_norm_workspace(rows, cols)
        return s
    H, K, D, it = case["heads"], case["kv_heads"], case["dim"], _IDX[case["ids"]]
    order = np.random.RandomState(seed % (1 << 32)).permutation(case["N"])
    nk, nq = (n[order] for n in _lengths(case))
    room = nk if case["queries"] == "all" else np.ceil(nk / (1.0 - case["room"])).astype(np.int64)

    def offsets(n):
        return torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(it).cuda()

    s |= {"q_offsets": offsets(nq), "k_offsets": offsets(room), "k_lengths": None, "most": (int(nq.max()), int(nk.max())), "bias": None, "bucket_map": None}
    Q, R = int(nq.sum()), int(room.sum())
    if case["queries"] == "all":
        s["q"], s["k"], s["v"] = normal(Q, H + 2 * K, D).to(io).split((H, K, K), 1)
    else:
        s["q"], s["k"], s["v"] = normal(Q, H, D).to(io), normal(R, K, D).to(io), normal(R, K, D).to(io)
        if case["room"]:
            s["k_lengths"] = torch.from_numpy(nk).to(it).cuda()
    if case["buckets"]:
        s["bias"], s["bucket_map"] = normal(H, case["buckets"], mul=0.5).to(io), _bucket_map(case)
    if case["op"] == "attention_backward":
        s["grad"] = normal(Q, H, D).to(io)
        s["out"], s["lse"] = _plain_attention(s, False)
    if own:
        s["workspace"] = s["tbe"].alloc_attention_workspace(case["N"], Q, R, H, K, D, buckets=case["buckets"], backward=case["op"] == "attention_backward")
    return s


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"layer_norm": _plain_norm, "layer_norm_backward": _plain_norm_backward}[op](s) if op.startswith("layer_norm") else _plain_attention(s, op == "attention_backward")
    tbe = s["tbe"]
    if op == "layer_norm":
        return tbe.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    if op == "layer_norm_backward":
        return tbe.layer_norm_backward(s["grad"], s["x"], s["weight"], s["mean"], s["rstd"], s["workspace"])
    how = {"causal": s["case"]["causal"], "k_lengths": s["k_lengths"], "bias": s["bias"], "bucket_map": s["bucket_map"]}
    if op == "attention":
        return tbe.attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], s["workspace"], **how)
    grads = tbe.attention_backward(s["grad"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["q_offsets"], s["k_offsets"], s["workspace"], **how)
    return grads if s["bias"] is not None else grads[:3]


def _plain_norm(s):
    x, io = s["x"].float(), s["x"].dtype
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = torch.rsqrt(x.square().mean(1) + EPS)
    return (x * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(io), mean, rstd


def _plain_norm_backward(s):
    dy, io, params = s["grad"].float(), s["x"].dtype, s["weight"].dtype
    xh = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
    return dx.to(io), (dy * xh).sum(0).to(params), dy.sum(0).to(params)


def _plain_attention(s, backward):
    """The operators on sequences padded to the longest, in 32 bits: every score is written to memory."""
    c = s["case"]
    N, H, K, D, (Lq, Lk) = c["N"], c["heads"], c["kv_heads"], c["dim"], s["most"]
    G, io, dev = H // K, s["q"].dtype, s["q"].device
    q0, k0 = s["q_offsets"][:-1].long(), s["k_offsets"][:-1].long()
    nq = s["q_offsets"][1:].long() - q0
    nk = s["k_lengths"].long() if s["k_lengths"] is not None else s["k_offsets"][1:].long() - k0
    i, j = torch.arange(Lq, device=dev), torch.arange(Lk, device=dev)
    has_q, has_k = i < nq[:, None], j < nk[:, None]
    at_q, at_k = (q0[:, None] + i) * has_q, (k0[:, None] + j) * has_k
    place = (nk - nq)[:, None] + i
    seen = has_q[:, :, None] & has_k[:, None, :]
    if c["causal"]:
        seen = seen & (j <= place[:, :, None])

    def padded(x, at, has):  # [N, heads, L, D]
        return (x[at].float() * has[:, :, None, None]).permute(0, 2, 1, 3).contiguous()

    def times(a, b):  # over the batch and the heads, in 32 bits
        return torch.bmm(a.reshape(N * K, -1, a.shape[-1]), b.reshape(N * K, -1, b.shape[-1])).reshape(N, -1, a.shape[2], b.shape[3])

    def grouped(x):  # the heads of a group one below the other
        return x.reshape(N, K, -1, x.shape[-1])

    scale = 1.0 / math.sqrt(D)
    q, k, v = padded(s["q"], at_q, has_q), padded(s["k"], at_k, has_k), padded(s["v"], at_k, has_k)
    x = times(grouped(q), k.transpose(2, 3)).reshape(N, H, Lq, Lk).mul_(scale)
    if s["bias"] is not None:
        far = c["far"]
        bucket = s["bucket_map"].long()[(place[:, :, None] - j).clamp_(-far, far) + far]
        x += s["bias"].float().t()[bucket].permute(0, 3, 1, 2)
    x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    lse = torch.log(total) + top
    p /= torch.where(total == 0, torch.ones_like(total), total)
    rows = at_q[has_q]

    def packed(x, to, at, has):  # [N, heads, L, D] to rows
        to[at[has]] = x.permute(0, 2, 1, 3)[has].to(to.dtype)
        return to

    if not backward:
        out = packed(times(grouped(p), v).reshape(N, H, Lq, D), torch.empty(s["q"].shape, dtype=io, device=dev), at_q, has_q)
        at_lse = torch.empty(H, s["q"].shape[0], device=dev)
        at_lse[:, rows] = lse[..., 0].permute(1, 0, 2)[:, has_q]
        return out, at_lse
    dy = padded(s["grad"], at_q, has_q)
    dv = times(grouped(p).transpose(2, 3), grouped(dy))
    ds = times(grouped(dy), v.transpose(2, 3)).reshape(N, H, Lq, Lk)
    ds -= (ds * p).sum(3, keepdim=True)
    ds *= p
    dq = times(grouped(ds), k).reshape(N, H, Lq, D).mul_(scale)
    dk = times(grouped(ds).transpose(2, 3), grouped(q)).mul_(scale)
    new = [torch.zeros(s[n].shape, dtype=io, device=dev) for n in "qkv"]
    grads = packed(dq, new[0], at_q, has_q), packed(dk, new[1], at_k, has_k), packed(dv, new[2], at_k, has_k)
    if s["bias"] is None:
        return grads
    # rows of the scores moved until a distance is one column, the columns added, and the distances' sums by bucket
    W = Lq + Lk
    moved = torch.nn.functional.pad(ds.flip(2), (0, Lq)).reshape(N, H, Lq * W)[..., :Lq * (W - 1)].reshape(N, H, Lq, W - 1)
    by_distance = moved.sum(2).permute(1, 0, 2).reshape(H, -1)  # column c of sequence n: key - query = c - (Lq - 1)
    distance = (nk - nq)[:, None] - (torch.arange(W - 1, device=dev) - (Lq - 1))
    bucket = s["bucket_map"].long()[distance.clamp_(-far, far) + far].reshape(-1)
    return (*grads, (by_distance @ torch.nn.functional.one_hot(bucket, c["buckets"]).float()).to(io))


def exact(case, seed):
    """The same from the definitions, sequence by sequence in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"].startswith("layer_norm"):
        x, w, b, n = s["x"].to(f64), s["weight"].to(f64), s["bias"].to(f64), case["cols"]
        mean = x.sum(1) / n
        var = ((x - mean[:, None]) ** 2).sum(1) / n
        if case["op"] == "layer_norm":
            return torch.addcmul(b, (x - mean[:, None]) / (var + EPS).sqrt()[:, None], w), mean, 1.0 / (var + EPS).sqrt()
        mean, rstd, dy = s["mean"].to(f64)[:, None], s["rstd"].to(f64)[:, None], s["grad"].to(f64)
        hat = (x - mean) * rstd
        along = (dy * w).sum(1, keepdim=True) / n + hat * (dy * w * hat).sum(1, keepdim=True) / n
        return rstd * (dy * w - along), (dy * hat).sum(0), dy.sum(0)
    H, K, D, far = case["heads"], case["kv_heads"], case["dim"], case["far"]
    backward = case["op"] == "attention_backward"
    qo, ko = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    ends = [a + n for a, n in zip(ko, s["k_lengths"].tolist())] if s["k_lengths"] is not None else ko[1:]
    out, lse = torch.zeros(s["q"].shape, dtype=f64, device="cuda"), torch.full((H, s["q"].shape[0]), -math.inf, dtype=f64, device="cuda")
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=f64, device="cuda") for n in "qkv")
    db = torch.zeros(H, max(1, case["buckets"]), dtype=f64, device="cuda")
    shared = torch.arange(H, device="cuda") // (H // K)
    for n in range(case["N"]):
        a, b, c, e = qo[n], qo[n + 1], ko[n], ends[n]
        if a == b or c == e:
            continue
        q, k, v = s["q"][a:b].to(f64).transpose(0, 1), s["k"][c:e].to(f64)[:, shared].transpose(0, 1), s["v"][c:e].to(f64)[:, shared].transpose(0, 1)
        apart = torch.arange(e - c - (b - a), e - c, device="cuda")[:, None] - torch.arange(e - c, device="cuda")
        x = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(D)
        if s["bias"] is not None:
            x = x + s["bias"].to(f64)[:, s["bucket_map"].long()[apart.clamp(-far, far) + far]]
        if case["causal"]:
            x = x.masked_fill(apart < 0, -math.inf)
        total = torch.logsumexp(x, 2)
        p = torch.exp(x - torch.where(total == -math.inf, torch.zeros_like(total), total)[:, :, None])
        del x
        out[a:b], lse[:, a:b] = torch.matmul(p, v).transpose(0, 1), total
        if not backward:
            continue
        dy = s["grad"][a:b].to(f64).transpose(0, 1)
        dv[c:e].index_add_(1, shared, torch.matmul(p.transpose(1, 2), dy).transpose(0, 1))
        ds = p * (torch.matmul(dy, v.transpose(1, 2)) - (dy * out[a:b].transpose(0, 1)).sum(2, keepdim=True))
        dq[a:b] = torch.matmul(ds, k).transpose(0, 1) / math.sqrt(D)
        dk[c:e].index_add_(1, shared, torch.matmul(ds.transpose(1, 2), q).transpose(0, 1) / math.sqrt(D))
        if s["bias"] is not None:
            nq, nk = b - a, e - c
            wide = torch.zeros(H, nq, nk + 2 * nq, dtype=f64, device="cuda")
            wide[:, :, nq:nq + nk] = ds
            # lines along which key - query stays the same, from key - query = -nq on
            lines = wide.as_strided((H, nq + nk, nq), (nq * (nk + 2 * nq), 1, nk + 2 * nq + 1)).sum(2)
            d = (nk - nq) - (torch.arange(nq + nk, device="cuda") - nq)
            db.index_add_(1, s["bucket_map"].long()[d.clamp(-far, far) + far], lines)
    if not backward:
        return out, lse
    return (dq, dk, dv, db) if s["bias"] is not None else (dq, dk, dv)
