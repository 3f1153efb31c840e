"""Attention over packed sequences from its definition, sequence by sequence in 64 bits, with bounds of what rounding may do to the
kernels' results.  Shared by the attention tests; not a test module itself.

Bounds.  u = 2^-24 rounds fp32 sums and products, t the operands' type (2^-8 bfloat16, 2^-11 binary16, 0 fp32).
  score        e_x = u ((dim + 8) |scale| sum_d |q k| + 4 |x| + 4 |bias|), its largest over the row
  probability  relative: 2 e_x + 16 u from the exponent, its function and the row's sum (nk more u), t where it is rounded
  out          sum_j P |v| (2 e_x + (nk + 24) u + t), and t of the result once more; binary16 probabilities also lose 2^-24 each
  dS           P (|dP - D| (2 e_x + 24 u) + u (dim + 4) (sum_d |dout v| + sum_d |dout out|) + t sum_d |dout out|), since D is taken
               from the rounded out; t of it where it is rounded
  gradients    the sums of those times |k|, |q|, |dout|, the sums' own u per term, and t of the result
Half a unit of binary16's subnormals (2^-25) is added for every rounded factor and result."""
import math

import torch

U = 2.0 ** -24
T = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}


def bucket_map(far, buckets, causal):
    """Nearest distances one bucket each, further ones by their logarithm; distances ahead share the other half."""
    out = []
    half = buckets if causal else max(1, buckets // 2)
    near = max(1, half // 2)
    for d in range(-far, far + 1):
        a = abs(d)
        b = a if a < near else min(half - 1, near + int(math.log(a / near) / math.log(max(far, near + 1) / near) * (half - near)))
        b = min(b, half - 1)
        out.append(min(buckets - 1, b + half) if d < 0 and not causal else b)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def reference(q, k, v, nq, nk, k0, *, causal, scale, bias=None, map_=None, dout=None):
    """nq, nk: queries and keys of every sequence; k0: its first key row.  Returns a dict of results and of their bounds ("~name")."""
    H, K, D = q.shape[1], k.shape[1], q.shape[2]
    f64, dev, t, tiny = torch.float64, q.device, T[q.dtype], TINY[q.dtype]
    shared = torch.arange(H, device=dev) // (H // K)
    r = {"out": torch.zeros(q.shape, dtype=f64, device=dev), "lse": torch.full((H, q.shape[0]), -math.inf, dtype=f64, device=dev)}
    r["~out"], r["~lse"] = torch.zeros_like(r["out"]), torch.zeros(H, q.shape[0], dtype=f64, device=dev)
    if dout is not None:
        for n, like in (("dq", q), ("dk", k), ("dv", v)):
            r[n], r["~" + n] = torch.zeros(like.shape, dtype=f64, device=dev), torch.zeros(like.shape, dtype=f64, device=dev)
        if bias is not None:
            r["dbias"], r["~dbias"] = torch.zeros(bias.shape, dtype=f64, device=dev), torch.zeros(bias.shape, dtype=f64, device=dev)
    a = 0
    for n, m, c in zip(nq, nk, k0):
        b = a + n
        if n and m:
            Q, Kk, V = (x.to(f64).transpose(0, 1) for x in (q[a:b], k[c:c + m][:, shared], v[c:c + m][:, shared]))
            d = torch.arange(m - n, m, device=dev)[:, None] - torch.arange(m, device=dev)
            x = Q @ Kk.transpose(1, 2) * scale
            e = ((D + 8) * abs(scale) * (Q.abs() @ Kk.abs().transpose(1, 2)) + 4 * x.abs()) * U
            if bias is not None:
                far = map_.numel() // 2
                at = map_.long()[d.clamp(-far, far) + far]
                bx = torch.where((at >= 0) & (at < bias.shape[1]), bias.to(f64)[:, at.clamp(0, bias.shape[1] - 1)], torch.zeros((), dtype=f64, device=dev))
                x = x + bx
                e = e + 4 * bx.abs().nan_to_num(posinf=0.0, neginf=0.0) * U + torch.where(bx == -math.inf, 0.0, 4 * x.abs().nan_to_num(posinf=0, neginf=0) * U)
            seen = (d >= 0) if causal else torch.ones_like(d, dtype=torch.bool)
            x = x.masked_fill(~seen, -math.inf)
            e = e.masked_fill(~seen, 0.0).nan_to_num(nan=0.0).amax(2, keepdim=True)
            lse = torch.logsumexp(x, 2)
            p = torch.exp(x - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)[..., None])
            rel = 2 * e + (m + 24) * U
            V0 = torch.where(torch.isfinite(V), V, torch.zeros_like(V))
            r["out"][a:b], r["lse"][:, a:b] = (p @ V0).transpose(0, 1), lse
            r["~out"][a:b] = ((p @ V0.abs()) * (rel + t) + t * (p @ V0).abs() + tiny * (1 + V0.abs().sum(1, keepdim=True))).transpose(0, 1)
            r["~lse"][:, a:b] = e[..., 0] + (m + 24) * U + 4 * U * lse.abs().nan_to_num(posinf=0, neginf=0)
            if dout is not None:
                dy = dout[a:b].to(f64).transpose(0, 1)
                o = r["out"][a:b].transpose(0, 1)
                dp, dsum, dmag = dy @ V.transpose(1, 2), (dy * o).sum(2, keepdim=True), (dy * o).abs().sum(2, keepdim=True)
                ds = p * (dp - dsum)
                raw = p * ((dp - dsum).abs() * rel + U * (D + 4) * (dy.abs() @ V.abs().transpose(1, 2) + dmag)) + p * (t * dmag + (dy.abs() * r["~out"][a:b].transpose(0, 1)).sum(2, keepdim=True))
                err = raw + t * ds.abs() + tiny
                perr = p * (rel + t) + tiny
                aK, aQ, aY = Kk.abs(), Q.abs(), dy.abs()
                for name, val, bound, terms in (("dv", p.transpose(1, 2) @ dy, perr.transpose(1, 2) @ aY + n * U * (p.transpose(1, 2) @ aY), n),
                                                ("dk", scale * (ds.transpose(1, 2) @ Q), abs(scale) * (err.transpose(1, 2) @ aQ + (n + 4) * U * (ds.abs().transpose(1, 2) @ aQ)), n)):
                    r[name][c:c + m].index_add_(1, shared, val.transpose(0, 1))
                    r["~" + name][c:c + m].index_add_(1, shared, (bound + H * U * val.abs()).transpose(0, 1))
                r["dq"][a:b] = (scale * (ds @ Kk)).transpose(0, 1)
                r["~dq"][a:b] = (abs(scale) * (err @ aK + (m + 4) * U * (ds.abs() @ aK))).transpose(0, 1)
                if bias is not None:
                    ok = (at >= 0) & (at < bias.shape[1])
                    r["dbias"].index_add_(1, at[ok], ds[:, ok])
                    r["~dbias"].index_add_(1, at[ok], (raw + (n + m + 64) * U * ds.abs())[:, ok])
        a = b
    if dout is not None:
        for n in ("dq", "dk", "dv"):
            r["~" + n] += t * r[n].abs() + tiny
        if bias is not None:
            tb = T[bias.dtype]
            r["~dbias"] += tb * r["dbias"].abs() + TINY[bias.dtype]
    return r


def check(got, ref, names, what):
    for g, n in zip(got, names):
        x, y, bound = g.double(), ref[n], ref["~" + n]
        same = (x == y) | (torch.isnan(x) & torch.isnan(y))
        err = (x - y).abs()
        bad = ~same & ~(err <= bound)
        assert not bool(bad.any()), (f"{what}: {n}: {int(bad.sum())} of {bad.numel()} over the bound, first at {bad.nonzero()[0].tolist()}: "
                                     f"{x[bad][0].item():.8g} for {y[bad][0].item():.8g} +- {bound[bad][0].item():.3g}")
