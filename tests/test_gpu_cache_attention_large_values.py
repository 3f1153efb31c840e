"""Attention over caches whose values come near fp32's largest number: results, being means of them, are finite, on every way the work is shared out;
beside them what does not see such values keeps its bits, and what is not a number reaches what it should.

Bounds: those of tests/attention_reference.py.  A probability is smaller by a power of two there, 2^-lift; its exponent is rounded at a size that is greater
by at most twice the lift (below 40): 64 u of every probability more, and 64 u of lse.  What is smaller than 2^-86 may be lost."""
import math

import pytest
import torch

from attention_reference import U, check, reference
from test_gpu_cache_attention import E4M3, I8, build, gen, run, values

pytestmark = pytest.mark.gpu
BIG = 240 * 2.0 ** 120   # (256 2^120, the next e4m3 code, is beyond fp32)


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def wanted(s, nq, nk, causal=True):
    k, v = values(s["cache"], "k"), values(s["cache"], "v")
    how = dict(causal=causal, scale=s["q"].shape[2] ** -0.5, bias=s["bias"], map_=s["bucket_map"])
    ref = reference(s["q"], k, v, nq, nk, s["k0"], **how)
    ref["~out"] += 64 * U * reference(s["q"], k, v.abs(), nq, nk, s["k0"], **how)["out"] + 2.0 ** -86
    ref["~lse"] += 64 * U
    return ref


def compare(tbe, s, nq, nk, what, causal=True):
    got = run(tbe, s, causal=causal)
    assert bool(got[0].isfinite().all()), what
    check(got, wanted(s, nq, nk, causal), ("out", "lse"), what)
    again = run(tbe, s, causal=causal)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def fill(tbe, s, v):
    """The cache's values, written: [rows, heads, dim]."""
    c = s["cache"]
    k = torch.randn(v.shape, generator=gen(v.shape[0]), device="cuda")
    tbe.cache_write(c, k, v.clamp(-BIG, BIG), torch.arange(len(v), device="cuda"))


SHAPES = [([1] * 3, [300, 40, 7], 4, 2, 32), ([1], [5000], 16, 2, 128), ([1, 1], [3000, 900], 3, 3, 64), ([61, 40], [1500, 800], 2, 1, 64), ([70, 3], [70, 3], 2, 2, 128),
          ([5, 33], [700, 4000], 8, 4, 48)]


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("buckets", [0, 16])
@pytest.mark.parametrize("causal", [True, False])
def test_near_the_largest_number(tbe, io, code, buckets, causal):
    for nq, nk, H, K, dim in SHAPES:
        s = build(tbe, gen(dim), nq, nk, nk, H, K, dim, io, code, buckets=buckets, causal=causal, poison=False)
        shape = s["cache"].k.shape
        g = gen(7)
        for kind in range(3):
            v = torch.rand(shape, generator=g, device="cuda") * 0.3 + 0.7   # of one sign
            if kind == 1:
                v *= torch.randint(0, 2, shape, generator=g, device="cuda") * 2.0 - 1.0
            v *= BIG
            if kind == 2:   # beside rows that are ordinary or small
                v *= torch.pow(10.0, -torch.randint(0, 3, (shape[0], shape[1], 1), generator=g, device="cuda") * 20.0)
            fill(tbe, s, v)
            compare(tbe, s, nq, nk, f"{H}/{K} {dim} {nq} {kind}", causal)


@pytest.mark.parametrize("code", [E4M3, I8])
def test_parts_that_leave_the_range_when_they_are_joined(tbe, code):
    """All scores 0, so that a run's sum is its keys times the value: at some of these sizes each run's is in range, and their sum is not."""
    for nk, H, K, dim, io in (([5000], 16, 2, 128, torch.bfloat16), ([9000, 300], 2, 2, 32, torch.float32), ([40_000], 4, 1, 64, torch.float32), ([2000] * 20, 8, 2, 64, torch.bfloat16)):
        nq = [1] * len(nk)
        s = build(tbe, gen(dim), nq, nk, nk, H, K, dim, io, code, poison=False)
        s["q"].zero_()
        for e in range(108, 128):
            v = torch.rand(s["cache"].k.shape, generator=gen(e), device="cuda") * 0.5 + 0.9375
            fill(tbe, s, v * 2.0 ** (e - 1))
            compare(tbe, s, nq, nk, f"{nk} 2^{e}")


@pytest.mark.parametrize("io", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("code", [E4M3, I8])
def test_those_that_do_not_see_them_keep_their_bits(tbe, io, code):
    """Large values at the last keys of a sequence: of the queries in one tile, those further back and other heads' are as they are without."""
    nq, nk = [9, 33], [400, 1000]
    s = build(tbe, gen(3), nq, nk, nk, 4, 2, 64, io, code, poison=False)
    clean = run(tbe, s)
    c = s["cache"]
    old = c.v_scales[1].clone()
    for n, key in ((0, 395), (1, 1390)):
        c.v_scales[1, key:key + 3] = 2.0 ** 120 if code == I8 else 2.0 ** 118
    got = run(tbe, s)
    c.v_scales[1] = old
    sees = torch.zeros(42, dtype=torch.bool, device="cuda")
    sees[4:9] = sees[32:] = True   # place nk - nq + i of query i
    assert torch.equal(got[0][~sees], clean[0][~sees]) and torch.equal(got[0][:, :2], clean[0][:, :2])
    if io != torch.float16:
        assert bool(got[0].isfinite().all()) and bool((got[0][sees][:, 2:].abs().amax(2) > 1e25).all())


def test_hidden_and_not_a_number_beside_them(tbe):
    for io in (torch.float32, torch.bfloat16):
        nq, nk = [33, 1], [500, 3000]
        s = build(tbe, gen(4), nq, nk, [510, 3010], 2, 2, 32, io, E4M3)   # (room of codes and scales that are not numbers)
        c = s["cache"]
        filled = torch.zeros(3520, dtype=torch.bool, device="cuda")
        filled[:500] = filled[510:3510] = True
        c.v_scales[:, filled] = 2.0 ** 119
        v = c.v.float()
        v[filled] = v[filled].clamp(-240, 240).abs() + 1
        c.v.view(torch.uint8)[filled] = v[filled].to(E4M3).view(torch.uint8)
        full = run(tbe, s)
        assert bool(full[0].isfinite().all())
        check(full, wanted(s, nq, nk), ("out", "lse"), "hidden")
        c.v.view(torch.uint8)[498, 1, 9] = 0x7F   # seen by the last two of the first sequence's queries
        c.v.view(torch.uint8)[510 + 2999, 0, 30] = 0xFF   # by the second's
        got = run(tbe, s)
        odd = torch.zeros_like(got[0], dtype=torch.bool)
        odd[31:33, 1, 9] = odd[33, 0, 30] = True
        assert bool(got[0][odd].isnan().all()) and torch.equal(got[0][~odd], full[0][~odd])


def test_a_scale_that_is_not_a_number_among_them(tbe):
    nq, nk = [1, 3], [600, 4000]
    s = build(tbe, gen(5), nq, nk, nk, 4, 2, 64, torch.bfloat16, I8, poison=False)
    s["cache"].v_scales.fill_(2.0 ** 120)
    s["cache"].v_scales[0, 600 + 17] = math.nan
    got = run(tbe, s)
    assert bool(got[0][1:, :2].isnan().all()) and bool(got[0][0].isfinite().all()) and bool(got[0][1:, 2:].isfinite().all())
    assert bool(got[1].isfinite().all())


def test_the_largest_numbers_read_as_infinite(tbe):
    """A code times its scale beyond fp32: from halfway between 240 and 256 times 2^120 on with e4m3, with i8 for fp32's largest number alone, whose quotient
    by 127 is rounded up."""
    top = torch.finfo(torch.float32).max
    x = torch.zeros(4, 1, 16, device="cuda")
    x[:, 0, 3] = torch.tensor([top, 248 * 2.0 ** 120, 0.0, 0.0], device="cuda")
    x[2, 0, 3] = torch.nextafter(x[1, 0, 3], torch.zeros((), device="cuda"))
    x[3, 0, 3] = torch.nextafter(x[0, 0, 3], torch.zeros((), device="cuda"))
    for code, want in ((E4M3, [math.inf, math.inf, 240 * 2.0 ** 120, math.inf]), (I8, [math.inf, None, None, None])):
        c = tbe.alloc_cache(4, 1, 16, code)
        slots = torch.arange(4, device="cuda")
        tbe.cache_write(c, x, -x, slots)
        k, v = tbe.cache_read(c, slots)
        for i, w in enumerate(want):
            got = k[i, 0, 3].item()
            assert v[i, 0, 3].item() == -got and (got == w if w is not None else math.isfinite(got) and abs(got / x[i, 0, 3].item() - 1) < 2.0 ** -22)
        assert bool((k[:, 0, 4:] == 0).all())


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("code", [E4M3, I8])
def test_small_values_keep_their_accuracy(tbe, io, code):
    """Values around 2^-90: probabilities of 2^-20 times them still have 24 bits above the last one of bfloat16's subnormal numbers, 2^-133."""
    for nq, nk, H, K, dim in SHAPES + [([1], [60_000], 2, 1, 32)]:
        s = build(tbe, gen(dim), nq, nk, nk, H, K, dim, io, code, poison=False)
        fill(tbe, s, torch.randn(s["cache"].k.shape, generator=gen(1), device="cuda") * 2.0 ** -90)
        got = run(tbe, s)
        ref = reference(s["q"], values(s["cache"], "k"), values(s["cache"], "v"), nq, nk, s["k0"], causal=True, scale=dim ** -0.5)
        check(got, ref, ("out", "lse"), f"{H}/{K} {dim} {nq}")
