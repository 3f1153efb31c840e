"""Attention and its gradients over batches of many short sequences, where 32 neighbouring rows share a wavefront whatever sequences they
are of: against the definition in 64 bits (tests/attention_reference.py derives the bounds), with runs of empty sequences, other numbers of
keys than of queries, every way the bias is met, and values that are not finite, which stay in their sequence."""
import math

import pytest
import torch

import attention_reference as R
from test_gpu_attention import TYPES, problem, refer, run
from test_gpu_attention_backward import NAMES, back, upstream

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def lengths(n, seed, most=40):
    """Mostly short, some empty, one run of 150 empty ones, a few longer than two tiles."""
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.exp(1.5 + torch.randn(n, generator=g)).round().clamp(0, most).long()
    x[torch.rand(n, generator=g) < 0.1] = 0
    x[n // 3:n // 3 + 150] = 0
    x[::97] = torch.randint(60, 140, (len(x[::97]),), generator=g)
    return x.tolist()


def both(tbe, p, what):
    dout = upstream(p)
    fwd = run(tbe, p)
    ref = refer(p, None, dout)
    R.check(fwd, ref, ("out", "lse"), what)
    got = back(tbe, p, dout, fwd)
    n = 4 if p["bias"] is not None else 3
    R.check(got[:n], ref, NAMES[:n], what)
    again = run(tbe, p), back(tbe, p, dout, fwd)
    assert all(torch.equal(a, b) for a, b in zip(fwd, again[0])) and all(torch.equal(a, b) for a, b in zip(got[:n], again[1][:n])), what
    assert not tbe.poll_index_error(), what


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [32, 24, 64, 128])
def test_short_sequences(tbe, io, D):
    n = lengths(420, D)
    for H, K in ((8, 8), (8, 2)):
        for causal, buckets, far in ((True, 16, 10), (False, 9, 200), (True, 0, 0)):
            both(tbe, problem(n, n, H, K, D, TYPES[io], causal=causal, buckets=buckets, far=far, ids=torch.int32 if causal else torch.int64), f"{io} {D} {H}/{K} {causal} {buckets}")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_other_numbers_of_keys(tbe, io):
    """Places that do not lie as the rows do: several turns over the keys in one wavefront, sequences without keys or without queries, more
    queries than keys."""
    g = torch.Generator()
    g.manual_seed(8)
    nq = lengths(400, 3)
    nk = [max(0, m + int(d)) for m, d in zip(nq, torch.randint(-6, 9, (len(nq),), generator=g))]
    for causal, buckets, far in ((True, 16, 10), (False, 9, 50), (True, 0, 0)):
        both(tbe, problem(nq, nk, 8, 4, 32, TYPES[io], causal=causal, buckets=buckets, far=far), f"{io} {causal} {buckets}")


def test_one_long_sequence_among_short_ones(tbe):
    n = [3] * 200 + [900] + [5] * 220
    both(tbe, problem(n, n, 8, 8, 32, torch.bfloat16, buckets=16, far=100), "long among short")


def test_what_is_not_finite_stays_in_its_sequence(tbe):
    n = [7, 9, 20, 5] * 110
    for io, D in (("f32", 32), ("bf16", 32), ("f16", 64)):
        p = problem(n, n, 8, 8, D, TYPES[io], buckets=4, far=6)
        dout, fwd = upstream(p), run(tbe, p)
        clean = back(tbe, p, dout, fwd)
        lo = sum(n[:41])                                     # a sequence of 9 between one of 7 and one of 20
        for what, x in (("v", p["v"]), ("k", p["k"]), ("q", p["q"])):
            keep = x[lo + 4, 3, 1].clone()
            x[lo + 4, 3, 1] = math.nan if what != "v" else math.inf
            got = run(tbe, p)
            grads = back(tbe, p, dout, got)
            x[lo + 4, 3, 1] = keep
            for a, b in zip((got[0], *grads[:3]), (fwd[0], *clean[:3])):
                assert torch.equal(a[:lo], b[:lo]) and torch.equal(a[lo + 9:], b[lo + 9:]) and torch.equal(a[lo:lo + 9, :3], b[lo:lo + 9, :3]), (io, what)
            assert not bool(torch.isfinite(got[0][lo + 4, 3]).all())
        dout[lo + 4, 3, 1] = math.inf
        grads = back(tbe, p, dout, fwd)
        for a, b in zip(grads[:3], clean[:3]):
            assert torch.equal(a[:lo], b[:lo]) and torch.equal(a[lo + 9:], b[lo + 9:])
        assert not bool(torch.isfinite(grads[2][lo + 4, 3]).all())


def test_offsets_that_do_not_fit_are_reported(tbe):
    n = [6] * 500
    p = problem(n, n, 8, 8, 32, torch.float32)
    dout, fwd = upstream(p), run(tbe, p)
    for which, at, by in (("q_offsets", 250, 100), ("k_offsets", 499, 40), ("q_offsets", 500, 6), ("k_offsets", 0, 1), ("k_offsets", 77, -500), ("q_offsets", 3, 1 << 40)):
        s = dict(p)
        s[which] = p[which].clone()
        s[which][at] += by
        out = torch.full_like(fwd[0], 7.0)
        run(tbe, s, out=out)
        assert tbe.poll_index_error(), (which, at)
        assert bool(torch.isfinite(out).all())
        back(tbe, s, dout, fwd)
        assert tbe.poll_index_error(), (which, at)
