"""Gradients of rows whose visible scores are all large in magnitude, where one fp32 number cannot hold both their maximum and the logarithm
of their sum: biases of the type's lowest value, and scores of 1e5.  The bounds do not grow with the bias.

Bounds.  The queries are so small that all scores of a row, its bias aside, lie within s = max |q . k| scale of 0, so that rounding
them at the bias's magnitude moves a score by 2 s at most and a probability by 4 s of itself; the rest is as derived in
tests/attention_reference.py, with e_x = u (dim + 8) s + 4 s u.  P moves by r = 4 s + 2 e_x + (nk + 24) u of itself (and t where it is rounded),
D = sum_j P_ij dP_ij by (2 r + 3 t) and (dim + nk + 4) u of the products' magnitudes, for it comes from P or from the out of the forward, which
rounds P and its result."""
import math

import pytest
import torch

import attention_reference as R
from test_gpu_attention import TYPES, problem, run
from test_gpu_attention_backward import NAMES, back, upstream

pytestmark = pytest.mark.gpu
SMALL = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -24, torch.float16: 2.0 ** -14}
# queries and keys of the sequences: on their own wavefronts, on shared ones, on tiles that a workgroup shares
LENGTHS = {"own": [40, 9, 33, 1, 64], "shared": [7, 9, 20, 5, 1, 70] * 60, "tiles": [500, 130, 330], "few tiles": [300, 40, 100, 1, 257]}


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def definition(p, dout):
    q, k, v, bias, map_ = p["q"], p["k"], p["v"], p["bias"], p["bucket_map"]
    H, K, D, f64, dev, u = q.shape[1], k.shape[1], q.shape[2], torch.float64, q.device, R.U
    t, tiny, scale = R.T[q.dtype], R.TINY[q.dtype], q.shape[2] ** -0.5
    shared = torch.arange(H, device=dev) // (H // K)
    r = {n: torch.zeros(x.shape, dtype=f64, device=dev) for n, x in (("dq", q), ("dk", k), ("dv", v))}
    if bias is not None:
        r["dbias"] = torch.zeros(bias.shape, dtype=f64, device=dev)
    r |= {"~" + n: torch.zeros_like(x) for n, x in r.items()}
    a = 0
    for n, m, c in zip(p["nq"], p["nk"], p["k0"]):
        Q, Kk, V, dy = (x.to(f64).transpose(0, 1) for x in (q[a:a + n], k[c:c + m][:, shared], v[c:c + m][:, shared], dout[a:a + n]))
        d = torch.arange(m - n, m, device=dev)[:, None] - torch.arange(m, device=dev)
        x = Q @ Kk.transpose(1, 2) * scale
        if bias is None:
            s, e = 0.0, (D + 8) * u * 0.0   # (whole numbers: these scores are exact, and all the same)
        else:
            s = float(x.abs().max())
            e = u * (D + 12) * s
            at = map_.long()[d.clamp(-(map_.numel() // 2), map_.numel() // 2) + map_.numel() // 2]
            x = x + bias.to(f64)[:, at].clamp(-1e30, 1e30)
        x = x.masked_fill((d < 0) if p["causal"] else torch.zeros_like(d, dtype=torch.bool), -math.inf)
        P = torch.softmax(x, 2)
        P = torch.where(P < 2.0 ** -126, torch.zeros_like(P), P)    # (what binary32 does not hold)
        rel = 4 * s + 2 * e + (m + 24) * u
        dP, mag = dy @ V.transpose(1, 2), dy.abs() @ V.abs().transpose(1, 2)
        Dsum, Dmag, Dall = (P * dP).sum(2, keepdim=True), (P * dP.abs()).sum(2, keepdim=True), (P * mag).sum(2, keepdim=True)
        dS = P * (dP - Dsum)
        raw = P * ((dP - Dsum).abs() * rel + (2 * rel + 3 * t) * Dall + (D + m + 4) * u * (mag + Dall) + tiny * dy.abs().sum(2, keepdim=True))
        err, perr = raw + t * dS.abs() + tiny, P * (rel + t) + tiny
        for name, val, bound in (("dv", P.transpose(1, 2) @ dy, perr.transpose(1, 2) @ dy.abs() + n * u * (P.transpose(1, 2) @ dy.abs())),
                                 ("dk", scale * (dS.transpose(1, 2) @ Q), scale * ((err + (n + 4) * u * dS.abs()).transpose(1, 2) @ Q.abs()))):
            r[name][c:c + m].index_add_(1, shared, val.transpose(0, 1))
            r["~" + name][c:c + m].index_add_(1, shared, (bound + H * u * val.abs()).transpose(0, 1))
        r["dq"][a:a + n] = (scale * (dS @ Kk)).transpose(0, 1)
        r["~dq"][a:a + n] = (scale * ((err + (m + 4) * u * dS.abs()) @ Kk.abs())).transpose(0, 1)
        if bias is not None:
            r["dbias"].index_add_(1, at.reshape(-1), dS.reshape(H, -1))
            r["~dbias"].index_add_(1, at.reshape(-1), (raw + (n + m + 64) * u * dS.abs()).reshape(H, -1))
        a += n
    for n in ("dq", "dk", "dv"):
        r["~" + n] += t * r[n].abs() + tiny
    if bias is not None:
        r["~dbias"] += R.T[bias.dtype] * r["dbias"].abs() + R.TINY[bias.dtype] + sum(p["nq"]) * u * r["~dbias"]
    return r


def agree(tbe, p, what):
    dout, fwd = upstream(p), run(tbe, p)
    got = back(tbe, p, dout, fwd)
    n = 4 if p["bias"] is not None else 3
    R.check(got[:n], definition(p, dout), NAMES[:n], what)
    assert all(torch.equal(a, b) for a, b in zip(got[:n], back(tbe, p, dout, fwd)[:n])), what


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_all_visible_scores_at_a_low_value(tbe, io, lengths):
    n, H = LENGTHS[lengths], 8 if lengths == "shared" else 2
    for D, K, causal, far in ((32, H, True, 200), (64, 1, True, 10), (128, H, False, 200)):
        p = problem(n, n, H, K, D, TYPES[io], buckets=8, far=far, causal=causal)
        p["q"] *= SMALL[TYPES[io]]
        for low in (torch.finfo(TYPES[io]).min, -1e9, -65504.0, -1e4, -300.0):
            if io == "f16" and low < -65504:
                continue
            p["bias"][:] = low
            agree(tbe, p, f"{io} {lengths} {D} {low}: all buckets")
            p["bias"][0, 3:] = 0.5      # rows that see a bucket of these have no other probabilities
            agree(tbe, p, f"{io} {lengths} {D} {low}: near buckets of one head")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_other_numbers_of_keys_at_a_low_value(tbe, io):
    for nq, nk, H in (([20, 3, 33] * 2, [90, 3, 200] * 2, 4), ([3, 7, 5, 9] * 90, [5, 7, 6, 12] * 90, 8), ([300, 200], [900, 210], 2)):
        p = problem(nq, nk, H, 2, 32, TYPES[io], buckets=8, far=30, room=[3] * len(nq) if H == 4 else None)
        p["q"] *= SMALL[TYPES[io]]
        p["bias"][:] = -1e9
        agree(tbe, p, f"{io} {nq[:3]}")


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lengths", list(LENGTHS))
@pytest.mark.parametrize("sign", [1, -1])
def test_large_equal_scores_without_a_bias(tbe, io, lengths, sign):
    """q . k scale = +-131072 for all pairs, which binary32 holds: every visible key counts the same."""
    n, H = LENGTHS[lengths], 8 if lengths == "shared" else 2
    p = problem(n, n, H, H, 64, TYPES[io])
    p["q"][:] = 64.0 * sign
    p["k"][:] = 256.0
    agree(tbe, p, f"{io} {lengths}")
