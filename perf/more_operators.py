"""The measured cases of the operators between a projection and the attention that follows it: heads normed and rotated by their positions, forward
and backward, and caches of one byte per element, written, read back and attended to.

  op        rotate | rotate_backward | cache_write | cache_read | cache_attention
rotate, rotate_backward
  rows, q_heads, k_heads, dim; q and k are column blocks of one matrix whose remaining columns are the values
  turned    elements of a head that are rotated, the first ones; layout: "half" (element j with j + turned / 2) | "pairs" (2 j with 2 j + 1)
  norm      heads are divided by their root mean square and multiplied by a weight first; params: type of the weights
  span      positions lie below this; stretch: the context is this many times the one that the frequencies are made for (1: as it is)
cache_write, cache_read
  cache     rows of the cache; rows: that many of them, in no order, are written or read; heads, dim; io: type of the rows
  code      "e4m3" | "i8"
cache_attention
  N         sequences, packed one after the other in the cache, with a share of `room` that no token has filled yet
  lengths   keys of a sequence: "fixed L" | "uniform lo hi" | "lognormal mu sigma cap" (the lengths' spread is the case's, their order the seed's)
  queries   the last so many tokens of a sequence (fewer where it is shorter) attend to its whole cache; 1 is a decoding step
  heads, kv_heads, dim, causal, io (q and out), code, ids (offsets and lengths); buckets, far: a bias by distance, 0: none
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-6
_IO = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_CODE = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
_IDX = {"i64": torch.int64, "i32": torch.int32}
_BYTES = {"i64": 8, "i32": 4, "f32": 4, "f16": 2, "bf16": 2}


def _turn(name, op, rows, q_heads, k_heads, dim, turned, layout, norm, io, params="f32", span=500, stretch=1.0, ids="i64"):
    return {"name": name, "op": op, "rows": rows, "q_heads": q_heads, "k_heads": k_heads, "dim": dim, "turned": turned, "layout": layout,
            "norm": norm, "io": io, "params": params, "span": span, "stretch": stretch, "ids": ids}


def _copy(name, op, cache, rows, heads, dim, io, code, ids="i64"):
    return {"name": name, "op": op, "cache": cache, "rows": rows, "heads": heads, "dim": dim, "io": io, "code": code, "ids": ids}


def _attend(name, N, lengths, heads, kv_heads, dim, io, code, queries=1, room=0.2, causal=True, buckets=0, far=128, ids="i64"):
    return {"name": name, "op": "cache_attention", "N": N, "lengths": lengths, "queries": queries, "room": room, "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "causal": causal, "io": io, "code": code, "ids": ids, "buckets": buckets, "far": far}


def listed():
    return [
        # the newest event of each user of a serving request: latency only
        _turn("rotate_request", "rotate", 32, 4, 4, 32, 32, "half", True, "f32", ids="i32"),
        # the tokens of a training batch, grouped heads, normed
        _turn("rotate_events", "rotate", 131_071, 16, 4, 128, 128, "half", True, "bf16", span=32_768),
        # part of each head in full precision, positions far beyond what the frequencies were made for
        _turn("rotate_far", "rotate", 60_001, 8, 8, 80, 32, "pairs", False, "f32", span=4_000_000, stretch=32.0),
        # the gradients of the training batch, both weights' among them
        _turn("rotate_events_backward", "rotate_backward", 65_537, 16, 4, 128, 128, "half", True, "bf16", span=32_768),
        # ... of part of each head, without a norm
        _turn("rotate_part_backward", "rotate_backward", 40_003, 12, 12, 64, 24, "half", False, "f16", span=8_192),
        # one new event for each user of a request goes into the users' caches
        _copy("write_request", "cache_write", 32_768, 32, 4, 32, "f32", "i8", ids="i32"),
        # whole prompts go into a cache with room left
        _copy("write_prompt", "cache_write", 250_000, 200_003, 8, 128, "bf16", "e4m3"),
        # some hundred tokens of a large cache are looked at again
        _copy("read_some", "cache_read", 100_000, 700, 4, 64, "f32", "e4m3", ids="i32"),
        # most of a cache goes back to the rows' type
        _copy("read_most", "cache_read", 150_000, 120_011, 8, 96, "bf16", "i8"),
        # one new event for each of a request's users against their short histories, with a bias by distance
        _attend("request_cache_step", 32, "lognormal 2 1 500", 4, 4, 32, "f32", "i8", buckets=32, ids="i32"),
        # one new event against very long histories, many heads on few keys
        _attend("long_history_step", 24, "uniform 2000 65536", 16, 2, 128, "bf16", "e4m3"),
        # a few dozen new events behind a middling history
        _attend("append_to_cache", 48, "uniform 100 4000", 8, 8, 64, "f16", "i8", queries=61, room=0.1, ids="i32"),
    ]


def draw(rng):
    def spread(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    op = rng.choice(("rotate", "rotate", "rotate_backward", "rotate_backward", "cache_write", "cache_read", "cache_attention", "cache_attention", "cache_attention"))
    io, ids, code = rng.choice(("f32", "f16", "bf16", "bf16")), rng.choice(("i64", "i32")), rng.choice(("e4m3", "i8"))
    if op.startswith("rotate"):
        k_heads = rng.choice((1, 2, 3, 4, 8))
        q_heads = k_heads * rng.choice((1, 1, 2, 3, 4))
        dim = rng.choice((16, 32, 40, 64, 64, 72, 80, 96, 100, 128, 128, 192, 256))
        turned = rng.choice((dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)))
        rows = int(spread(1, (1.6e8 if op == "rotate" else 8.0e7) / ((q_heads + k_heads) * dim)))
        case = _turn("", op, rows, q_heads, k_heads, dim, turned // 2 * 2, rng.choice(("half", "half", "pairs")), rng.random() < 0.6, io,
                     rng.choice(("f32", io)), int(spread(100, 1.0e7)), rng.choice((1.0, 1.0, 4.0, 32.0)), ids)
    elif op != "cache_attention":
        heads, dim = rng.choice((1, 2, 3, 4, 8, 16)), 16 * rng.randint(1, 8)
        cache = int(spread(8, 1.5e8 / (heads * dim)))
        case = _copy("", op, cache, max(1, int(cache * rng.choice((rng.random(), 1.0, 0.01)))), heads, dim, io, code, ids)
    else:
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
        dim = rng.choice((16, 32, 32, 48, 64, 64, 80, 96, 128, 128))
        queries = rng.choice((1, 1, 1, int(spread(2, 200))))
        longest = spread(20, 60_000 if queries == 1 else 6_000)
        shape = rng.choice(("fixed %d" % longest, "uniform %d %d" % (longest / spread(1, 30), longest), "lognormal %.2f 1 %d" % (math.log(longest / 12 + 1), longest)))
        N, most = max(1, int(spread(1, 4000))), int(shape.split()[-1])
        asking = min(most, queries)
        # pairs of a padded batch, their operations, and the tokens
        while N > 1 and (N * heads * most * asking > 6.0e8 or N * heads * most * asking * dim > 4.0e10 or N * most * kv_heads * dim > 2.0e8):
            N = N * 2 // 3
        while heads > kv_heads and heads * most * asking > 6.0e8:
            heads -= kv_heads
        case = _attend("", N, shape, heads, kv_heads, dim, io, code, queries, rng.choice((0.0, 0.15)), rng.random() < 0.8, rng.choice((0, 0, 16, 48)),
                       rng.choice((32, 128, 500)), ids)
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
    return n, np.minimum(n, case["queries"])


def work(case):
    w, i = _BYTES[case["io"]], _BYTES[case["ids"]]
    if case["op"].startswith("rotate"):
        heads, params = case["q_heads"] + case["k_heads"], 2 * case["dim"] * _BYTES[case["params"]] if case["norm"] else 0
        n = case["rows"] * heads * case["dim"]
        rest = case["rows"] * i + case["turned"] // 2 * 8
        turned = case["rows"] * heads * case["turned"]
        if case["op"] == "rotate":
            return {"bytes": 2 * n * w + params + rest, "flops": 3 * turned + (4 * n if case["norm"] else 0)}
        return {"bytes": (3 if case["norm"] else 2) * n * w + 2 * params + rest, "flops": 3 * turned + (10 * n if case["norm"] else 0)}
    if case["op"] != "cache_attention":
        n = 2 * case["rows"] * case["heads"]
        return {"bytes": n * case["dim"] * (w + 1) + 4 * n + case["rows"] * i, "flops": (3 if case["op"] == "cache_write" else 1) * n * case["dim"]}
    nk, nq = _lengths(case)
    pairs = int((nq * nk - (nq * (nq - 1) // 2 if case["causal"] else 0)).sum()) * case["heads"]
    q, k = int(nq.sum()) * case["heads"], int(nk.sum()) * case["kv_heads"]
    return {"bytes": 2 * q * case["dim"] * w + 4 * q + 2 * k * (case["dim"] + 4) + case["heads"] * case["buckets"] * w, "flops": 4 * case["dim"] * pairs}


def _frequencies(case):
    """Radians per position of every pair, 64 bits: a geometric series from 1 down to 1 / 10000; for a context that is longer than the one it was made
    for, those that turn less than once in that context divided by the stretch, those that turn 32 times and more as they are, between them a
    line in the number of turns."""
    half = case["turned"] // 2
    f = 10_000.0 ** (-np.arange(half) / half)
    turns = np.clip((case["span"] / case["stretch"] * f / (2 * np.pi) - 1.0) / 31.0, 0.0, 1.0)
    return torch.from_numpy(f if case["stretch"] == 1.0 else turns * f + (1.0 - turns) * f / case["stretch"]).cuda()


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


def _plain_codes(x, code):
    """One byte for every element of [rows, heads, dim], and the scale of every row and head."""
    x = x.float()
    top = x.abs().amax(2)
    if code == "e4m3":  # the least power of two with which the largest magnitude is at most 448 = 0.875 * 2 ^ 9
        fraction, exponent = torch.frexp(top)
        exponent = (exponent - torch.where(fraction <= 0.875, 9, 8)).clamp(min=-126)
        exponent = torch.where(top == 0, torch.zeros_like(exponent), exponent)
        return torch.ldexp(x, -exponent[:, :, None]).to(torch.float8_e4m3fn), torch.ldexp(torch.ones_like(top), exponent)
    scale = torch.where(top == 0, torch.ones_like(top), (top / 127.0).clamp(min=2.0 ** -126))
    return torch.round(x.double() / scale.double()[:, :, None]).to(torch.int8), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    io, it = _IO[case["io"]], _IDX[case["ids"]]

    def normal(*shape, mul=1.0, add=0.0):
        return torch.randn(*shape, generator=g, device="cuda").mul_(mul).add_(add)

    def rows(n, heads, dim):  # some of a head's elements are large in every row
        x = normal(n, heads, dim)
        return x.mul_(torch.exp(normal(heads, dim, mul=0.7))).to(io)

    s = {"case": case}
    if own:
        from paper_2508_03854_amd import TBE, Cache
        s["tbe"] = TBE([16], [8])
    if case["op"].startswith("rotate"):
        n, H, K, D = case["rows"], case["q_heads"], case["k_heads"], case["dim"]
        s["positions"] = torch.randint(0, case["span"], (n,), generator=g, device="cuda").to(it)
        s["frequencies"], s["amplitude"] = _frequencies(case), 0.1 * math.log(case["stretch"]) + 1.0
        s["q"], s["k"], _ = rows(n, H + 2 * K, D).split((H, K, K), 1)
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"], s["k_weight"] = (normal(D, mul=0.2, add=1.0).to(_IO[case["params"]]) for _ in range(2))
        if case["op"] == "rotate_backward":
            s["grad_q"], s["grad_k"] = normal(n, H, D).to(io), normal(n, K, D).to(io)
            if own:
                s["workspace"] = s["tbe"].alloc_rotate_workspace(n, H, K, D)
        return s
    if case["op"] == "cache_attention":
        N, H, K, D = case["N"], case["heads"], case["kv_heads"], case["dim"]
        order = np.random.RandomState(seed % (1 << 32)).permutation(N)
        nk, nq = (n[order] for n in _lengths(case))
        room = np.ceil(nk / (1.0 - case["room"])).astype(np.int64)

        def offsets(n):
            return torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(it).cuda()

        Q, R = int(nq.sum()), int(room.sum())
        s |= {"q": normal(Q, H, D).to(io), "q_offsets": offsets(nq), "k_offsets": offsets(room), "k_lengths": torch.from_numpy(nk).to(it).cuda(),
              "most": (int(nq.max()), int(nk.max())), "bias": None, "bucket_map": None}
        (k, ks), (v, vs) = (_plain_codes(rows(R, K, D), case["code"]) for _ in range(2))
        if case["buckets"]:
            s["bias"], s["bucket_map"] = normal(H, case["buckets"], mul=0.5).to(io), _bucket_map(case)
        if own:
            s["workspace"] = s["tbe"].alloc_cache_attention_workspace(N, Q, R, H, K, D, buckets=case["buckets"])
    else:
        C, n, K, D = case["cache"], case["rows"], case["heads"], case["dim"]
        s["slots"] = torch.randperm(C, generator=g, device="cuda")[:n].to(it)
        if case["op"] == "cache_write":
            s["k"], s["v"] = rows(n, 2 * K, D).split((K, K), 1)
            k = v = torch.zeros(C, K, D, device="cuda").to(_CODE[case["code"]])
            ks = vs = torch.ones(C, K, device="cuda")
        else:
            (k, ks), (v, vs) = (_plain_codes(rows(C, K, D), case["code"]) for _ in range(2))
    k, ks, v, vs = k.clone(), ks.t().contiguous(), v.clone(), vs.t().contiguous()  # codes [rows, heads, dim], scales [heads, rows]
    s["cache"] = Cache(k, v, ks, vs) if own else (k, v, ks, vs)
    return s


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"rotate": _plain_rotate, "rotate_backward": _plain_rotate_backward, "cache_write": _plain_write, "cache_read": _plain_read,
                "cache_attention": _plain_attention}[op](s)
    tbe = s["tbe"]
    if op.startswith("rotate"):
        how = {"interleaved": c["layout"] == "pairs", "amplitude": s["amplitude"], "norm": c["norm"], "eps": EPS, "q_weight": s["q_weight"], "k_weight": s["k_weight"]}
        if op == "rotate":
            return tbe.rotate_heads(s["q"], s["k"], s["positions"], s["frequencies"], **how)
        grads = tbe.rotate_heads_backward(s["grad_q"], s["grad_k"], s["positions"], s["frequencies"], s["workspace"], q=s["q"], k=s["k"], **how)
        return grads if c["norm"] else grads[:2]
    if op == "cache_write":
        tbe.cache_write(s["cache"], s["k"], s["v"], s["slots"])
        return s["cache"].k, s["cache"].v, s["cache"].k_scales, s["cache"].v_scales
    if op == "cache_read":
        return tbe.cache_read(s["cache"], s["slots"], dtype=_IO[c["io"]])
    return tbe.cache_attention(s["q"], s["cache"], s["q_offsets"], s["k_offsets"], s["workspace"], causal=c["causal"], k_lengths=s["k_lengths"],
                               bias=s["bias"], bucket_map=s["bucket_map"])


def _plain_turn(x, s, back):
    """The rotation of [rows, heads, dim], or its transpose, in 32 bits; its angles in 64."""
    half, pairs = s["case"]["turned"] // 2, s["case"]["layout"] == "pairs"
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = ((t * s["amplitude"]).float()[:, None] for t in (torch.cos(angle), torch.sin(-angle if back else angle)))
    y = x.clone()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_rotate(s):
    def one(x, weight):
        io, x = x.dtype, x.float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(2, keepdim=True) + EPS) * weight.float()
        return _plain_turn(x, s, False).to(io)
    return one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])


def _plain_rotate_backward(s):
    def one(dy, x, weight):
        g = _plain_turn(dy.float(), s, True)
        if weight is None:
            return (g.to(dy.dtype),)
        x = x.float()
        r = torch.rsqrt(x.square().mean(2, keepdim=True) + EPS)
        h, u = x * r, g * weight.float()
        return (r * (u - h * (u * h).mean(2, keepdim=True))).to(dy.dtype), (g * h).sum((0, 1), dtype=torch.float64).to(weight.dtype)
    q, k = one(s["grad_q"], s["q"], s["q_weight"]), one(s["grad_k"], s["k"], s["k_weight"])
    return tuple(t for two in zip(q, k) for t in two)


def _plain_write(s):
    for x, codes, scales in ((s["k"], s["cache"][0], s["cache"][2]), (s["v"], s["cache"][1], s["cache"][3])):
        new, scale = _plain_codes(x, s["case"]["code"])
        codes.view(torch.uint8)[s["slots"]] = new.view(torch.uint8)
        scales[:, s["slots"]] = scale.t()
    return s["cache"]


def _plain_rows(s, code, at, io):
    """The cache's rows `at`, as what their codes stand for."""
    codes, scales = s["cache"][code], s["cache"][code + 2]
    return (codes.view(torch.uint8)[at].view(codes.dtype).float() * scales.t()[at][..., None]).to(io)


def _plain_read(s):
    return _plain_rows(s, 0, s["slots"], _IO[s["case"]["io"]]), _plain_rows(s, 1, s["slots"], _IO[s["case"]["io"]])


def _plain_attention(s):
    """The operator on sequences padded to the longest, in 32 bits: the cache's values and every score are written to memory."""
    c = s["case"]
    N, H, K, D, (Lq, Lk) = c["N"], c["heads"], c["kv_heads"], c["dim"], s["most"]
    io, dev = s["q"].dtype, s["q"].device
    q0, k0 = s["q_offsets"][:-1].long(), s["k_offsets"][:-1].long()
    nq, nk = s["q_offsets"][1:].long() - q0, s["k_lengths"].long()
    i, j = torch.arange(Lq, device=dev), torch.arange(Lk, device=dev)
    has_q, has_k = i < nq[:, None], j < nk[:, None]
    at_q, at_k = (q0[:, None] + i) * has_q, (k0[:, None] + j) * has_k
    place = (nk - nq)[:, None] + i
    seen = has_q[:, :, None] & has_k[:, None, :]
    if c["causal"]:
        seen = seen & (j <= place[:, :, None])

    def times(a, b):  # over the batch and the key heads, in 32 bits
        return torch.bmm(a.reshape(N * K, -1, a.shape[-1]), b.reshape(N * K, -1, b.shape[-1])).reshape(N, H, Lq, -1)

    q = (s["q"][at_q].float() * has_q[:, :, None, None]).permute(0, 2, 1, 3).contiguous()  # [N, H, Lq, D]
    k, v = ((_plain_rows(s, n, at_k.reshape(-1), torch.float32).reshape(N, Lk, K, D) * has_k[:, :, None, None]).permute(0, 2, 1, 3) for n in (0, 1))
    x = times(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D))
    if s["bias"] is not None:
        far = c["far"]
        bucket = s["bucket_map"].long()[(place[:, :, None] - j).clamp_(-far, far) + far]
        x += s["bias"].float().t()[bucket].permute(0, 3, 1, 2)
    x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    y = times(p / torch.where(total == 0, torch.ones_like(total), total), v.contiguous())
    # from padded rows to packed ones; what stands for no query goes to a row behind the last, which is left out
    Q = s["q"].shape[0]
    to = torch.where(has_q, q0[:, None] + i, Q).reshape(-1)
    out = torch.zeros(Q + 1, H, D, dtype=io, device=dev)
    out[to] = y.permute(0, 2, 1, 3).reshape(-1, H, D).to(io)
    all_lse = torch.full((H, Q + 1), -math.inf, device=dev)
    all_lse[:, to] = lse.permute(1, 0, 2).reshape(H, -1)
    return out[:Q], all_lse[:, :Q]


def exact(case, seed):
    """The same from the definitions in 64 bits: rotations as products of complex numbers, their gradients by differentiation, codes by counting the
    format's steps, attention sequence by sequence."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"].startswith("rotate"):
        half, D = case["turned"] // 2, case["dim"]
        angle = s["positions"].to(f64)[:, None, None] * s["frequencies"]
        turn = torch.polar(torch.full_like(angle, s["amplitude"]), angle)

        def forward(x, w):
            if w is not None:
                x = x / (x.square().sum(2, keepdim=True) / D + EPS).sqrt() * w
            part = x[..., :2 * half]
            part = part.unflatten(2, (half, 2)) if case["layout"] == "pairs" else part.unflatten(2, (2, half)).transpose(2, 3)
            z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
            z = z if case["layout"] == "pairs" else z.transpose(2, 3)
            return torch.cat((z.flatten(2), x[..., 2 * half:]), 2)

        results, weights = [], []
        for n in "qk":
            x, w = s[n].to(f64), s[n + "_weight"]
            w = None if w is None else w.to(f64)
            if case["op"] == "rotate":
                results.append(forward(x, w))
                continue
            leaves = [x.requires_grad_()] + ([] if w is None else [w.requires_grad_()])
            grads = torch.autograd.grad(forward(x, w), leaves, s["grad_" + n].to(f64))
            results.append(grads[0])
            weights += grads[1:]
        return (*results, *weights)
    cache = s["cache"] if not own else (s["cache"].k, s["cache"].v, s["cache"].k_scales, s["cache"].v_scales)
    if case["op"] == "cache_write":
        codes, scales = [], []
        for x, old in ((s["k"], cache[0]), (s["v"], cache[1])):
            x, y, z = x.to(f64), old.to(f64), torch.ones(case["heads"], case["cache"], dtype=f64, device="cuda")
            top = x.abs().amax(2, keepdim=True)
            if case["code"] == "e4m3":
                scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)))
                scale = torch.where(top > 448.0 * scale, 2 * scale, torch.where(top <= 224.0 * scale, scale / 2, scale))  # (a logarithm next to a whole number)
                x = x / scale
                step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
                x = torch.round(x / step) * step
            else:
                scale = top / 127.0
                x = torch.round(x / scale.float().to(f64))
            y[s["slots"].long()], z[:, s["slots"].long()] = x, scale[..., 0].t()
            codes.append(y)
            scales.append(z)
        return (*codes, *scales)
    at = slice(None) if case["op"] == "cache_attention" else s["slots"].long()
    k, v = ((codes.to(f64) * scales.to(f64).t()[..., None])[at] for codes, scales in (cache[0::2], cache[1::2]))
    if case["op"] == "cache_read":
        return k, v
    H, far = case["heads"], case["far"]
    qo, ko, nk = s["q_offsets"].tolist(), s["k_offsets"].tolist(), s["k_lengths"].tolist()
    out, lse = torch.zeros(s["q"].shape, dtype=f64, device="cuda"), torch.full((H, s["q"].shape[0]), -math.inf, dtype=f64, device="cuda")
    shared = torch.arange(H, device="cuda") // (H // case["kv_heads"])
    for n in range(case["N"]):
        a, b, c, e = qo[n], qo[n + 1], ko[n], ko[n] + nk[n]
        apart = torch.arange(e - c - (b - a), e - c, device="cuda")[:, None] - torch.arange(e - c, device="cuda")
        x = torch.matmul(s["q"][a:b].to(f64).transpose(0, 1), k[c:e].permute(1, 2, 0)[shared].contiguous()) / math.sqrt(case["dim"])
        if s["bias"] is not None:
            x = x + s["bias"].to(f64)[:, s["bucket_map"].long()[apart.clamp(-far, far) + far]]
        if case["causal"]:
            x = x.masked_fill(apart < 0, -math.inf)
        lse[:, a:b] = torch.logsumexp(x, 2)
        out[a:b] = torch.matmul(torch.softmax(x, 2), v[c:e].transpose(0, 1)[shared].contiguous()).transpose(0, 1)
    return out, lse
