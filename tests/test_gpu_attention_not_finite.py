"""Gradients of attention beside values that are not finite: by the definition, over the pairs that see each other alone, some elements of the
sequence's results are not finite, and the kernels' are so exactly there; all others are, bit by bit, what they are without these values
(those of its own sequence too, unless the value takes a key out of a softmax)."""
import math

import pytest
import torch

from test_gpu_attention import TYPES, problem, run
from test_gpu_attention_backward import NAMES, back, upstream

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def over_seen(x, y, seen):
    """sum_j x[i, j] y[j, :] over the pairs that are seen: what is not seen is left out, whatever it is."""
    return torch.where(seen[..., None], x[..., None] * y, torch.zeros((), dtype=y.dtype, device=y.device)).sum(1)


def definition(p, dout, s):
    """Of sequence s: where its results are finite."""
    q0, c, n, m = sum(p["nq"][:s]), p["k0"][s], p["nq"][s], p["nk"][s]
    q, k, v, f64 = p["q"], p["k"], p["v"], torch.float64
    H, K, D = q.shape[1], k.shape[1], q.shape[2]
    r = {"dq": torch.zeros(n, H, D, dtype=f64, device=q.device), "dk": torch.zeros(m, K, D, dtype=f64, device=q.device),
         "dv": torch.zeros(m, K, D, dtype=f64, device=q.device)}
    if p["bias"] is not None:
        r["dbias"] = torch.zeros(p["bias"].shape, dtype=f64, device=q.device)
    d = torch.arange(m - n, m, device=q.device)[:, None] - torch.arange(m, device=q.device)
    seen = d >= 0 if p["causal"] else torch.ones_like(d, dtype=torch.bool)
    for h in range(H):
        kh = h // (H // K)
        Q, dy, Kk, V = q[q0:q0 + n, h].to(f64), dout[q0:q0 + n, h].to(f64), k[c:c + m, kh].to(f64), v[c:c + m, kh].to(f64)
        x = (Q[:, None] * Kk).sum(2) * D ** -0.5
        if p["bias"] is not None:
            far = p["bucket_map"].numel() // 2
            at = p["bucket_map"].long()[d.clamp(-far, far) + far]
            x = x + p["bias"][h].to(f64)[at]
        x = torch.where(seen, x, torch.full((), -INF, dtype=f64, device=q.device))
        P = torch.softmax(x, 1)
        P = torch.where(seen.any(1)[:, None], P, torch.zeros_like(P))
        dP = torch.where(seen, (dy[:, None] * V).sum(2), torch.zeros_like(x))
        dS = P * (dP - (P * dP).sum(1, keepdim=True))
        r["dq"][:, h] = over_seen(dS, Kk, seen)
        r["dk"][:, kh] += over_seen(dS.t(), Q, seen.t())
        r["dv"][:, kh] += over_seen(P.t(), dy, seen.t())
        if p["bias"] is not None:
            r["dbias"][h].index_add_(0, at[seen], dS[seen])
    return {n: torch.isfinite(t) for n, t in r.items()}


def agree(tbe, p, s, row, what, head=1, col=3):
    """Every operand in turn has an element of sequence s that is not finite."""
    H, K = p["q"].shape[1], p["k"].shape[1]
    dout, q0, k0 = upstream(p), sum(p["nq"][:s]), p["k0"][s]
    fwd = run(tbe, p)
    clean = back(tbe, p, dout, fwd)
    for name, x, at, value in (("v", p["v"], k0, INF), ("v", p["v"], k0, NAN), ("k", p["k"], k0, NAN), ("k", p["k"], k0, INF), ("k", p["k"], k0, -INF),
                               ("q", p["q"], q0, NAN), ("dout", dout, q0, INF), ("dout", dout, q0, NAN)):
        h = head if x.shape[1] == H else head // (H // K)
        keep = x[at + row, h, col].clone()
        x[at + row, h, col] = value
        got = back(tbe, p, dout, run(tbe, p))
        finite = definition(p, dout, s)
        x[at + row, h, col] = keep
        for n, a, b in zip(NAMES, got, clean):
            if a is None:
                continue
            expect = torch.ones_like(a, dtype=torch.bool)
            if n == "dbias":
                expect = finite[n]
            else:
                lo = q0 if n == "dq" else k0
                expect[lo:lo + finite[n].shape[0]] = finite[n]
            said = f"{what}: {n} with {name} {value}"
            assert torch.equal(torch.isfinite(a), expect), f"{said}: {int((torch.isfinite(a) != expect).sum())} of {a.numel()}, {int((torch.isfinite(a) & ~expect).sum())} of these finite"
            if name == "k" and abs(value) == INF and n != "dbias":
                # a score of -infinity takes the key out of a row's softmax: the row's other probabilities are not what they were
                expect[lo:lo + finite[n].shape[0]] = False
            if n != "dbias":
                assert torch.equal(a[expect], b[expect]), f"{said}: {int((a[expect] != b[expect]).sum())} others changed"


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,H,K", [([200, 70], 2, 1), ([500, 330, 600], 2, 1), ([30, 20], 4, 1), ([20, 45] * 3, 2, 2), ([7, 9, 20, 5, 70, 3] * 75, 8, 8)])
def test_values_that_are_hidden_beside_such_that_are_seen(tbe, io, n, H, K):
    """A value that all queries of a sequence see, and one that the later ones see, both not finite, in different elements: either
    reaches the results that see it, and no others."""
    for D in (32, 64, 128):
        for far, buckets in ((0, 0), (20, 8)):
            p = problem(n, n, H, K, D, TYPES[io], buckets=buckets, far=far)
            clean = run(tbe, p)
            for s in (0, 1):
                q0, later = sum(n[:s]), n[s] // 2 + 3
                v = p["v"].clone()
                v[q0, 0, 3], v[q0 + later, 0, 1] = INF, NAN
                got = run(tbe, dict(p, v=v))
                expect = torch.ones_like(clean[0], dtype=torch.bool)
                expect[q0:q0 + n[s], :H // K, 3] = False
                expect[q0 + later:q0 + n[s], :H // K, 1] = False
                assert torch.equal(torch.isfinite(got[0]), expect), (D, far, s, int((torch.isfinite(got[0]) != expect).sum()))
                assert torch.equal(got[0][expect], clean[0][expect]) and torch.equal(got[1], clean[1]), (D, far, s)


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_sequences_that_share_wavefronts(tbe, io, causal):
    n = [7, 9, 20, 5, 70, 3] * 75
    for D in (32, 64) if io == "f32" else (32,):
        for buckets in (0, 4):
            p = problem(n, n, 8, 8, D, TYPES[io], buckets=buckets, far=6, causal=causal)
            agree(tbe, p, 67, 4, f"{D} {buckets}", 3)       # a sequence of 9 between one of 7 and one of 20
            agree(tbe, p, 70, 40, f"{D} {buckets} 70", 3)   # one of 70


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_own_wavefronts_and_shared_tiles(tbe, io, D):
    """Sequences on their own wavefronts, and on tiles that a workgroup shares; D = 128 has the latter in both kernels of the backward only beside
    tables of many distances.  Heads of a group one after the other, other numbers of keys than of queries."""
    for n, H, K, s, row in (([40, 100, 33], 2, 1, 1, 60), ([20, 9, 31, 70], 4, 2, 2, 4), ([500, 130, 330], 2, 1, 0, 301), ([700, 450], 2, 2, 1, 77)):
        for causal, buckets, far in ((True, 0, 0), (True, 8, 20), (True, 8, 1024), (False, 8, 20)):
            agree(tbe, problem(n, n, H, K, D, TYPES[io], buckets=buckets, far=far, causal=causal), s, row, f"{n} {causal} {buckets} {far}")
    for nq, nk, s, row in (([33, 20], [150, 60], 0, 25), ([200, 300], [260, 310], 1, 199), ([70, 150], [30, 100], 1, 66)):
        agree(tbe, problem(nq, nk, 2, 1, D, TYPES[io], buckets=8, far=20), s, row, f"{nq} {nk}")


def test_sequences_that_share_wavefronts_in_one_kernel(tbe):
    """Heads whose queries share wavefronts and whose keys do not."""
    n = [7, 9, 20, 5, 70, 3] * 75
    for io, D in (("f32", 128), ("f16", 64), ("bf16", 64), ("bf16", 128)):
        for causal, buckets in ((True, 0), (True, 4), (False, 4)):
            p = problem(n, n, 8, 8, D, TYPES[io], buckets=buckets, far=6, causal=causal)
            agree(tbe, p, 67, 4, f"{io} {D} {buckets}", 3)
            agree(tbe, p, 70, 40, f"{io} {D} {buckets} 70", 3)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_beside_scores_at_a_low_value(tbe, io):
    """Rows that find their maxima and sums again meet values that are not finite on the way."""
    for n, H, K, s, row, head in (([40, 100, 33], 2, 1, 1, 60, 1), ([500, 130, 330], 2, 1, 0, 301, 1), ([7, 9, 20, 5, 70, 3] * 75, 8, 8, 67, 4, 3)):
        for causal in (True, False):
            p = problem(n, n, H, K, 32, TYPES[io], buckets=4, far=10, causal=causal)
            p["q"] *= 2.0 ** -24
            p["bias"][:] = -1e9
            agree(tbe, p, s, row, f"{n[:3]} {causal}", head)
