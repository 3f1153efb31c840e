"""Caches of one byte an element: rows written and read back, against the formats' definitions in 64 bits; slots in any order, below zero and beyond the
cache; every type and address of the rows; ties, tiny, huge and not finite heads; what is not written keeps its bytes; streams, graphs, refusals.

Codes and scales are exact: scale and code are determined by the rows (ties to even), so they are compared for equality.  Reading back is one
product in fp32 and one rounding to the rows' type: within 2^-24 of the value, and half a unit in the last place of the type more."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
E4M3, I8 = torch.float8_e4m3fn, torch.int8
IO = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def coded(x, code):
    """Codes (as numbers) and scales of [rows, heads, dim], from the formats' definitions in 64 bits."""
    x = x.double()
    top = x.abs().amax(2)
    odd = ~torch.isfinite(x).all(2)
    top = torch.where(odd | (top == 0), torch.ones_like(top), top)
    if code == E4M3:
        e = torch.tensor([[max(-126, next(e for e in range(math.frexp(t)[1] - 12, 200) if t <= math.ldexp(448.0, e))) for t in r] for r in top.tolist()],
                         dtype=torch.float64, device=x.device).view(top.shape)
        e = torch.where(x.abs().amax(2) == 0, torch.zeros_like(e), e)
        scale = torch.exp2(e)
        y = x / scale[..., None]
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        c = torch.round(y / step) * step
    else:
        scale = torch.where(x.abs().amax(2) == 0, torch.ones_like(top), (top / 127).float().clamp(min=2.0 ** -126).double())
        c = torch.round(x / scale[..., None])
    c = torch.where(odd[..., None], torch.zeros_like(c), c)
    return c, torch.where(odd, torch.full_like(scale, math.nan), scale)


def numbers(codes):
    return codes.to(torch.float32).double() if codes.dtype == E4M3 else codes.double()


def same(a, b):
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def rows(g, n, heads, dim, dtype, spread=1.0):
    x = torch.randn(n, heads, dim, generator=g, device="cuda") * torch.exp(spread * torch.randn(n, heads, 1, generator=g, device="cuda"))
    return x.to(dtype)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def bits(cache):
    return [t.view(torch.uint8).clone() for t in (cache.k, cache.v)] + [t.view(torch.int32).clone() for t in (cache.k_scales, cache.v_scales)]


@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("dtype", IO)
@pytest.mark.parametrize("index", [torch.int64, torch.int32])
def test_write_and_read(tbe, code, dtype, index):
    for n, places, heads, dim in ((1, 1, 1, 16), (7, 20, 3, 32), (33, 33, 4, 48), (100, 300, 8, 64), (65, 70, 5, 80), (40, 41, 2, 96), (19, 64, 16, 112), (257, 500, 8, 128),
                                  (3, 9, 33, 128), (2, 5, 1000, 16), (5000, 6000, 1, 16)):
        g = gen(n * 7 + dim)
        k, v = rows(g, n, heads, dim, dtype), rows(g, n, heads, dim, dtype)
        cache = tbe.alloc_cache(places, heads, dim, code)
        for t in (cache.k, cache.v):
            t.view(torch.uint8).fill_(0x31)
        slots = torch.randperm(places, generator=g, device="cuda")[:n].to(index)
        if n > 3:
            slots[2] = -1
        before = bits(cache)
        tbe.cache_write(cache, k, v, slots)
        keep = torch.ones(places, dtype=torch.bool, device="cuda")
        keep[slots[slots >= 0].long()] = False
        after = bits(cache)
        for a, b in zip(before[:2], after[:2]):
            assert torch.equal(a[keep], b[keep])
        for a, b in zip(before[2:], after[2:]):
            assert torch.equal(a[:, keep], b[:, keep])
        there, at = slots >= 0, slots[slots >= 0].long()
        values = []
        for x, codes, scales in ((k, cache.k, cache.k_scales), (v, cache.v, cache.v_scales)):
            c, s = coded(x[there], code)
            got = numbers(codes.view(torch.uint8)[at].view(code))
            assert torch.equal(got, c), f"{n} {heads} {dim}: {int((got != c).sum())} codes differ"
            assert torch.equal(scales.t()[at].double(), s)
            values.append(torch.zeros(x.shape, dtype=torch.float64, device="cuda"))
            values[-1][there] = c * s[..., None]
        for out_type in IO:
            for got, want in zip(tbe.cache_read(cache, slots, dtype=out_type), values):
                ok = (got.double() - want).abs() <= (2.0 ** -24 + HALF[out_type] * 1.001) * want.abs() + TINY[out_type]
                if out_type == torch.float16:
                    ok |= (want.abs() >= 65504) & (got.abs().float() >= 65504)
                assert bool(ok.all())
        assert not tbe.poll_index_error()


@pytest.mark.parametrize("code", [E4M3, I8])
def test_ties_and_edges(tbe, code):
    """Every tie of the codes and its two neighbours in fp32, at several scales; the largest of a head on either side of a power of two."""
    if code == E4M3:
        grid = torch.arange(127, dtype=torch.uint8).view(E4M3).double()
        mids = (grid[1:] + grid[:-1]) / 2
    else:
        mids = torch.arange(127, dtype=torch.float64) + 0.5
        mids[-1] = 126.5
    for mul in (1.0, 2.0 ** -20, 3.0, 1.1, 2.0 ** 40, 1e-30, 0.7 * 2.0 ** -118):
        top = (448.0 if code == E4M3 else 127.0) * mul
        x = torch.zeros(3 * len(mids), 16, dtype=torch.float32)
        m = (mids * mul).float()
        for i, y in enumerate((m, torch.nextafter(m, torch.tensor(math.inf)), torch.nextafter(m, torch.tensor(0.0)))):
            x[i * len(mids):(i + 1) * len(mids), 0], x[i * len(mids):(i + 1) * len(mids), 5] = y, -y
        x[:, 9] = top
        x = x.view(-1, 1, 16).cuda()
        cache = tbe.alloc_cache(len(x), 1, 16, code)
        tbe.cache_write(cache, x, -x, torch.arange(len(x), device="cuda"))
        c, s = coded(x, code)
        assert torch.equal(numbers(cache.k), c) and torch.equal(numbers(cache.v), -c) and torch.equal(cache.k_scales.t().double(), s)
    tops = [448.0, 448.00003, 447.99997, 449, 480, 512, 256, 255.99998, 224, 224.00002, 3.4e38, 1e-38, 1e-44, 1.4e-45, 0.0, 2.0 ** -126, 448 * 2.0 ** -126, 1e38]
    x = torch.zeros(len(tops), 1, 32)
    x[:, 0, 31] = torch.tensor(tops)
    x[:, 0, 0] = -torch.tensor(tops) / 3
    cache = tbe.alloc_cache(len(tops), 1, 32, code)
    tbe.cache_write(cache, x.cuda(), x.cuda(), torch.arange(len(tops), device="cuda"))
    c, s = coded(x.cuda(), code)
    assert torch.equal(numbers(cache.k), c) and torch.equal(cache.k_scales.t().double(), s)


@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("dtype", IO)
def test_heads_that_are_not_finite(tbe, code, dtype):
    g = gen(3)
    k = rows(g, 6, 3, 48, dtype)
    v = k.clone()
    for r, bad in ((0, math.inf), (2, -math.inf), (5, math.nan)):
        k[r, 1, 17 * r % 48] = bad
    cache = tbe.alloc_cache(6, 3, 48, code)
    tbe.cache_write(cache, k, v, torch.arange(6, device="cuda"))
    for x, codes, scales in ((k, cache.k, cache.k_scales), (v, cache.v, cache.v_scales)):
        c, s = coded(x, code)
        assert torch.equal(numbers(codes), c) and same(scales.t().double(), s)
    got = tbe.cache_read(cache, torch.arange(6, device="cuda"), dtype=dtype)
    odd = torch.zeros(6, 3, dtype=torch.bool, device="cuda")
    odd[[0, 2, 5], 1] = True
    assert torch.equal(got[0].isnan().all(2), odd) and not bool(got[0][~odd].isnan().any()) and bool(torch.isfinite(got[1]).all())


def test_rows_at_any_address_and_strided_caches(tbe):
    g = gen(4)
    for dtype in IO:
        n, heads, dim = 21, 3, 48
        flat = torch.randn(n * 400 + 1, generator=g, device="cuda").to(dtype)
        k, v = flat[1:].as_strided((n, heads, dim), (400, 61, 1)), flat[1:].as_strided((n, heads, dim), (400, 61, 1), flat[1:].storage_offset() + 190)
        slots = torch.randperm(30, generator=g, device="cuda")[:n]
        want = tbe.alloc_cache(30, heads, dim)
        tbe.cache_write(want, k.contiguous(), v.contiguous(), slots)
        from paper_2508_03854_amd import Cache
        both = torch.full((30, 2, heads, dim + 16), 0x55, dtype=torch.uint8, device="cuda")
        by_head = torch.full((heads, 30, dim), 0x55, dtype=torch.uint8, device="cuda")
        for ck, cv in ((both[:, 0, :, :dim].view(E4M3), both[:, 1, :, 16:].view(E4M3)), (by_head.transpose(0, 1).view(E4M3), by_head.clone().transpose(0, 1).view(E4M3))):
            cache = Cache(ck, cv, torch.ones(heads, 30, device="cuda"), torch.ones(heads, 30, device="cuda"))
            tbe.cache_write(cache, k, v, slots)
            for a, b in ((cache.k, want.k), (cache.v, want.v)):
                assert torch.equal(a.view(torch.uint8)[slots], b.view(torch.uint8)[slots])
            assert torch.equal(cache.k_scales, want.k_scales) and torch.equal(cache.v_scales, want.v_scales)
            ref = tbe.cache_read(want, slots, dtype=dtype)
            wide = torch.full((n, heads, dim + 3), 7.0, dtype=dtype, device="cuda")
            got = tbe.cache_read(cache, slots, k_out=wide[..., 1:dim + 1], v_out=torch.empty_like(ref[1]))
            assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
            assert bool((wide[..., 0] == 7).all()) and bool((wide[..., dim + 1:] == 7).all())
        assert bool((both[:, 0, :, dim:] == 0x55).all()) and bool((both[:, 1, :, :16] == 0x55).all())


def test_bad_slots_are_left_out_and_reported(tbe):
    g = gen(5)
    k = rows(g, 4, 2, 16, torch.float32)
    for index in (torch.int64, torch.int32):
        cache = tbe.alloc_cache(10, 2, 16, I8)
        before = bits(cache)
        tbe.cache_write(cache, k, k, torch.tensor([10, -5, 2 ** 31 - 1, -2 ** 31], dtype=index, device="cuda"))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(before, bits(cache)))
        assert tbe.poll_index_error() and not tbe.poll_index_error()
        tbe.cache_write(cache, k, k, torch.arange(4, device="cuda", dtype=index))
        got = tbe.cache_read(cache, torch.tensor([1, 10, -1, 1, 3], dtype=index, device="cuda"))
        assert bool((got[0][1:3] == 0).all()) and torch.equal(got[0][0], got[0][3]) and bool((got[0][4] != 0).any())
        assert tbe.poll_index_error()
        tbe.cache_read(cache, torch.tensor([-1], dtype=index, device="cuda"))
        assert not tbe.poll_index_error()
    none = k[:0]
    tbe.cache_write(cache, none, none, torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert tbe.cache_read(cache, torch.zeros(0, dtype=torch.int64, device="cuda"))[0].shape == (0, 2, 16)


def test_places_beyond_two_to_the_32nd_byte(tbe):
    """A cache of 4.4e9 bytes: the last rows."""
    places = (1 << 32) // 2048 + 100_000
    cache = tbe.alloc_cache(places, 16, 128, I8)
    g = gen(6)
    k, v = rows(g, 3, 16, 128, torch.bfloat16), rows(g, 3, 16, 128, torch.bfloat16)
    slots = torch.tensor([places - 1, places - 3, 5], device="cuda")
    tbe.cache_write(cache, k, v, slots)
    c, s = coded(k, I8)
    assert torch.equal(numbers(cache.k[slots]), c) and torch.equal(cache.k_scales.t()[slots].double(), s)
    assert int((cache.k_scales != 1).sum()) == 48 and int(cache.k[places - 2].abs().sum()) == 0
    got = tbe.cache_read(cache, slots)
    assert torch.equal(got[0].double(), (c.float() * s.float()[..., None]).double())


def test_on_a_stream_and_in_a_graph(tbe):
    g = gen(7)
    k, v, slots = rows(g, 64, 4, 64, torch.bfloat16), rows(g, 64, 4, 64, torch.bfloat16), torch.randperm(100, generator=g, device="cuda")[:64]
    cache = tbe.alloc_cache(100, 4, 64)
    out = [torch.empty_like(k), torch.empty_like(v)]

    def work(stream=None):
        tbe.cache_write(cache, k, v, slots, stream=stream)
        tbe.cache_read(cache, slots, k_out=out[0], v_out=out[1], stream=stream)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    work(s)
    s.synchronize()
    want = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for n in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), n
        k.mul_(1.25), v.add_(k)
        work()
        torch.cuda.synchronize()
        want = [t.clone() for t in out]


def test_refusals(tbe):
    from paper_2508_03854_amd import Cache, TbeError, binding as B
    cache = tbe.alloc_cache(8, 2, 32)
    k, slots = torch.randn(3, 2, 32, device="cuda"), torch.arange(3, device="cuda")
    ones = torch.ones(2, 8, device="cuda")
    for bad, kind in ((lambda: tbe.cache_write(cache, k, k[:2], slots), ValueError), (lambda: tbe.cache_write(cache, k, k.half(), slots), ValueError),
                      (lambda: tbe.cache_write(cache, k[:2], k[:2], slots), ValueError), (lambda: tbe.cache_write(cache, k[:, :1], k[:, :1], slots), ValueError),
                      (lambda: tbe.cache_write(cache, k.double(), k.double(), slots), TypeError), (lambda: tbe.cache_write(cache, k, k, slots.float()), TypeError),
                      (lambda: tbe.cache_write(cache, k.cpu(), k, slots), ValueError), (lambda: tbe.cache_write(cache, k, k, slots.cpu()), ValueError),
                      (lambda: tbe.cache_read(cache, slots.float()), TypeError), (lambda: tbe.cache_read(cache, slots, k_out=k[:2]), ValueError),
                      (lambda: tbe.cache_read(cache, slots, k_out=k, v_out=k.half()), ValueError), (lambda: tbe.cache_read(cache, slots, dtype=torch.int8), TypeError),
                      (lambda: Cache(cache.k, cache.v.view(I8), ones, ones), TypeError), (lambda: Cache(k, k, ones, ones), TypeError),
                      (lambda: Cache(cache.k, cache.v[:7], ones, ones), ValueError), (lambda: Cache(cache.k, cache.v, ones[:1], ones), ValueError),
                      (lambda: Cache(cache.k, cache.v, ones.t(), ones), ValueError), (lambda: Cache(cache.k, cache.v, ones.double(), ones), TypeError),
                      (lambda: Cache(cache.k.cpu(), cache.v.cpu(), ones, ones), ValueError), (lambda: tbe.alloc_cache(8, 2, 32, torch.uint8), TypeError)):
        with pytest.raises(kind):
            bad()
    u8 = torch.zeros(4096, dtype=torch.uint8, device="cuda").view(I8)

    def of(heads, dim, stride, off=0, head=None):
        t = u8[off:].as_strided((4, heads, dim), (stride, dim if head is None else head, 1), off)
        return Cache(t, t, torch.ones(heads, 4, device="cuda"), torch.ones(heads, 4, device="cuda"))

    for c, status in ((of(2, 24, 48), B.ESHAPE), (of(1, 8, 16), B.ESHAPE), (of(1, 144, 144), B.ESHAPE), (of(2, 32, 72), B.EINVAL), (of(2, 32, 64, 8), B.EINVAL),
                      (of(2, 32, 16), B.EINVAL), (of(2, 32, 64, 0, 16), B.EINVAL)):
        x = torch.zeros(1, c.k.shape[1], c.k.shape[2], device="cuda")
        for call in (lambda: tbe.cache_write(c, x, x, slots[:1]), lambda: tbe.cache_read(c, slots[:1])):
            with pytest.raises(TbeError) as e:
                call()
            assert e.value.status == status
    flat = torch.zeros(32, device="cuda")
    with pytest.raises(TbeError):   # one element written by several rows
        tbe.cache_read(cache, slots, k_out=flat.expand(3, 2, 32), v_out=torch.empty(3, 2, 32, device="cuda"))
