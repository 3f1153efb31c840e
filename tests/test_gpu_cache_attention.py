"""Attention over caches of one byte an element, against the definition in 64 bits on the values that the codes stand for: both codes, every type of
q, head sizes and groups, lengths from none to long ones, room, causal or not, bias by distance; the ways the work is shared out (wavefronts on their own, parts
of the keys, many units of queries, sequences that are much longer than the average); rows that see nothing; what is not finite; streams, graphs, refusals.

Bounds: those of tests/attention_reference.py.  The kernels' products are exact in q and the codes (its products round once, u each), a scale is one rounding
more of the score (of the 4 |x| there), and a probability times its value's scale is rounded no more than a probability there."""
import math

import pytest
import torch

from attention_reference import bucket_map, check, reference

pytestmark = pytest.mark.gpu
E4M3, I8 = torch.float8_e4m3fn, torch.int8
IO = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def values(cache, which):
    codes, scales = (cache.k, cache.k_scales) if which == "k" else (cache.v, cache.v_scales)
    return codes.to(torch.float32).double() * scales.t().double()[..., None]


def build(tbe, g, nq, nk, room, H, K, dim, io, code, *, index=torch.int64, buckets=0, far=40, causal=True, poison=True):
    """q, a filled cache and offsets; the cache's room holds NaN codes and NaN scales."""
    Q, R = sum(nq), sum(room)
    q = torch.randn(Q, H, dim, generator=g, device="cuda").to(io)
    cache = tbe.alloc_cache(R, K, dim, code)
    if R:
        tbe.cache_write(cache, torch.randn(R, K, dim, generator=g, device="cuda"), torch.randn(R, K, dim, generator=g, device="cuda") * 1.5, torch.arange(R, device="cuda"))
    k0 = [sum(room[:i]) for i in range(len(room))]
    if poison:
        for c, n, r in zip(k0, nk, room):
            for t in (cache.k, cache.v):
                t.view(torch.uint8)[c + n:c + r] = 0x7F
            for t in (cache.k_scales, cache.v_scales):
                t[:, c + n:c + r] = math.nan
    off = lambda n: torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=index, device="cuda")  # noqa: E731
    s = {"q": q, "cache": cache, "q_offsets": off(nq), "k_offsets": off(room), "k_lengths": torch.tensor(nk, dtype=index, device="cuda"), "k0": k0}
    s["bias"] = torch.randn(H, buckets, generator=g, device="cuda").to(io) if buckets else None
    s["bucket_map"] = bucket_map(far, buckets, causal) if buckets else None
    s["ws"] = tbe.alloc_cache_attention_workspace(len(nq), Q, R, H, K, dim, buckets=buckets)
    s["ws"].fill_(255)
    return s


def run(tbe, s, **how):
    return tbe.cache_attention(s["q"], s["cache"], s["q_offsets"], s["k_offsets"], s["ws"], k_lengths=s["k_lengths"], bias=s["bias"], bucket_map=s["bucket_map"], **how)


def compare(tbe, s, nq, nk, what, causal=True, scale=None):
    got = run(tbe, s, causal=causal, scale=scale)
    ref = reference(s["q"], values(s["cache"], "k"), values(s["cache"], "v"), nq, nk, s["k0"], causal=causal, scale=s["q"].shape[2] ** -0.5 if scale is None else scale,
                    bias=s["bias"], map_=s["bucket_map"])
    check(got, ref, ("out", "lse"), what)
    again = run(tbe, s, causal=causal, scale=scale)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    assert not tbe.poll_index_error()
    return got


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("buckets", [0, 16])
def test_single_tokens(tbe, io, code, buckets):
    for H, K, dim in ((1, 1, 16), (4, 4, 32), (8, 2, 48), (6, 3, 64), (16, 2, 128), (12, 1, 96), (32, 1, 80), (5, 5, 112)):
        for nk in ([1], [40, 1, 33, 64, 7, 128, 90], [3000, 5], [0, 700, 256, 257, 1023, 0, 1, 300], [5000]):
            nq = [1] * len(nk)
            room = [n + i % 4 for i, n in enumerate(nk)]
            s = build(tbe, gen(dim + len(nk)), nq, nk, room, H, K, dim, io, code, buckets=buckets, index=torch.int32)
            compare(tbe, s, nq, nk, f"{H}/{K} {dim} {nk}")


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("buckets", [0, 16])
def test_several_queries(tbe, io, code, causal, buckets):
    """Queries on either side of a tile of columns, more than keys, none; units of queries beyond those that go with a part."""
    for H, K, dim in ((2, 2, 32), (4, 1, 64), (3, 3, 128), (8, 4, 48)):
        for nq, nk in (([5, 31, 32, 33], [9, 31, 400, 1000]), ([61, 61, 40], [1500, 61, 800]), ([0, 3, 70, 1], [50, 2, 60, 0]), ([1, 200, 0, 1], [900, 2000, 300, 0]),
                       ([150], [333]), ([2, 2, 2, 130, 2, 2, 2, 2], [300, 400, 500, 3000, 270, 256, 260, 280])):
            s = build(tbe, gen(dim), nq, nk, [n + 3 for n in nk], H, K, dim, io, code, buckets=buckets, causal=causal)
            compare(tbe, s, nq, nk, f"{H}/{K} {dim} {nq} {nk}", causal)


@pytest.mark.parametrize("code", [E4M3, I8])
def test_many_sequences(tbe, code):
    """Short caches, and so many units of queries that each wavefront has its own; longer ones among them."""
    g = gen(1)
    nk = [int(x) for x in torch.exp(2.0 + torch.randn(3000, generator=g, device="cuda")).clamp(0, 400)]
    nk[7], nk[2999] = 0, 1500
    nq = [1] * 3000
    s = build(tbe, g, nq, nk, nk, 8, 4, 32, torch.bfloat16, code)
    compare(tbe, s, nq, nk, "short")
    nq, nk = [40] * 80, [200 + 17 * (i % 30) for i in range(80)]
    s = build(tbe, g, nq, nk, nk, 32, 32, 32, torch.float16, code, buckets=16)
    compare(tbe, s, nq, nk, "many units")


@pytest.mark.parametrize("code", [E4M3, I8])
def test_caches_that_are_filled_to_a_small_part(tbe, code):
    """Fewer tiles of keys than there is room for: the keys are shared out by what is there."""
    for nq, nk, room, H, K, dim in (([1] * 4, [40, 0, 1, 33], [8192] * 4, 8, 2, 128), ([1, 1], [90, 5000], [60_000, 9000], 4, 4, 32), ([40, 3], [64, 70], [6000, 6000], 2, 1, 64),
                                    ([1], [33], [100_000], 16, 1, 64), ([1] * 3, [0, 0, 0], [4000] * 3, 2, 2, 48)):
        s = build(tbe, gen(21), nq, nk, room, H, K, dim, torch.bfloat16, code, buckets=0)
        compare(tbe, s, nq, nk, f"{nk} of {room}")


def test_many_caches_shared_out_evenly(tbe):
    """More sequences than a workgroup has lanes, in one run or several; some of them empty."""
    nk = [(37 * i * i + 11 * i) % 900 for i in range(601)]
    nk[5] = nk[300] = nk[600] = 0
    for code, io, nq, H, K, dim in ((E4M3, torch.bfloat16, [1] * 601, 1, 1, 128), (I8, torch.float32, [i % 3 for i in range(601)], 2, 2, 32)):
        s = build(tbe, gen(25), nq, nk, [n + 2 for n in nk], H, K, dim, io, code)
        compare(tbe, s, nq, nk, "even")


def test_many_queries_of_many_heads(tbe):
    """More units of queries of a sequence than workgroups that share its keys; so many that each has all keys to itself."""
    for nq, nk, H, K, dim in (([700], [1000], 32, 8, 32), ([4200], [600], 32, 32, 32), ([900, 3], [901, 400], 16, 16, 64)):
        s = build(tbe, gen(27), nq, nk, nk, H, K, dim, torch.bfloat16, E4M3)
        compare(tbe, s, nq, nk, f"{nq}")


def test_largest_tables_of_distances(tbe):
    for H, K, dim, far in ((4, 1, 128, 1024), (8, 2, 32, 700), (3, 3, 64, 1024), (4, 2, 64, 0)):
        for nq, nk in (([1, 1, 1], [3000, 900, 40]), ([33, 2], [1500, 2100])):
            for causal in (True, False):
                s = build(tbe, gen(26), nq, nk, nk, H, K, dim, torch.bfloat16, E4M3, buckets=20, far=far, causal=causal)
                compare(tbe, s, nq, nk, f"{H} {dim} {far} {nk}", causal)


def test_uneven_queries_where_the_average_is_one(tbe):
    """As many queries as sequences, but not one each: short caches, and long ones."""
    for nk in ([100, 30, 200, 64, 10], [3000, 300, 900, 2000, 100]):
        nq = [3, 0, 1, 1, 0]
        s = build(tbe, gen(22), nq, nk, nk, 4, 2, 64, torch.float16, I8)
        compare(tbe, s, nq, nk, f"{nq} {nk}")
    nq, nk = [64] + [0] * 63, [200] + [90] * 63
    s = build(tbe, gen(23), nq, nk, nk, 4, 2, 64, torch.bfloat16, E4M3)
    compare(tbe, s, nq, nk, "all of them one's")


def test_places_beyond_two_to_the_32nd_byte(tbe):
    """The last sequence of a cache of 4.5e9 bytes, the first one of which has 2.2e6 keys."""
    from paper_2508_03854_amd import Cache
    first, last, H, dim = (1 << 32) // 2048 + 100_000, 300, 16, 128
    g = gen(24)
    k, v = (torch.zeros(first + last, H, dim, dtype=I8, device="cuda") for _ in range(2))
    k[first:] = torch.randint(-127, 128, (last, H, dim), generator=g, device="cuda", dtype=torch.int32).to(I8)
    v[first:] = torch.randint(-127, 128, (last, H, dim), generator=g, device="cuda", dtype=torch.int32).to(I8)
    v[first - 1] = 127   # (the first sequence's last key)
    scales = torch.full((H, first + last), 0.01, device="cuda")
    cache = Cache(k, v, scales, scales)
    q = torch.randn(2, H, dim, generator=g, device="cuda").to(torch.bfloat16)
    qo, ko = torch.tensor([0, 1, 2], device="cuda"), torch.tensor([0, first, first + last], device="cuda")
    out, lse = tbe.cache_attention(q, cache, qo, ko, tbe.alloc_cache_attention_workspace(2, 2, first + last, H, H, dim))
    ref = reference(q[1:], k[first:].double() * 0.01, v[first:].double() * 0.01, [1], [last], [0], causal=True, scale=dim ** -0.5)
    scale32 = float(torch.tensor(0.01)) / 0.01 - 1   # (fp32's 0.01)
    ref["~out"] += abs(scale32) * (1 + ref["out"].abs()) * 4 + 1e-6
    ref["~lse"] += abs(scale32) * 4 * ref["lse"].abs() + 1e-6
    check((out[1:], lse[:, 1:]), ref, ("out", "lse"), "last")
    assert (lse[:, 0].double() - math.log(first)).abs().max() <= 1e-5   # all scores 0: every key the same
    assert (out[0].double() * first - 1.27).abs().max() <= 1.27 * 2.0 ** -7


def test_long_cache(tbe):
    for code, io, H, K, dim in ((E4M3, torch.bfloat16, 16, 2, 128), (I8, torch.float32, 4, 4, 64), (E4M3, torch.float16, 3, 1, 32)):
        nk = [100_003, 260]
        s = build(tbe, gen(2), [1, 2], nk, nk, H, K, dim, io, code, poison=False)
        compare(tbe, s, [1, 2], nk, "long")


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.7])
def test_scales_of_the_scores(tbe, scale):
    for io in IO:
        s = build(tbe, gen(3), [1, 4], [300, 50], [300, 60], 4, 2, 32, io, E4M3)
        compare(tbe, s, [1, 4], [300, 50], f"scale {scale}", scale=scale)


def test_without_lengths_and_strided(tbe):
    """Offsets alone; q and out column blocks of wider matrices, the cache's codes by head."""
    from paper_2508_03854_amd import Cache
    g = gen(4)
    nq, nk = [1, 3, 2], [500, 20, 300]
    s = build(tbe, g, nq, nk, nk, 4, 2, 64, torch.bfloat16, E4M3, poison=False)
    want = run(tbe, s)
    c = s["cache"]
    by_head = [t.view(torch.uint8).transpose(0, 1).contiguous().transpose(0, 1).view(E4M3) for t in (c.k, c.v)]
    wide = torch.full((6, 9, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.randn(6, 12, 64, generator=g, device="cuda").to(torch.bfloat16)
    q[:, 4:8] = s["q"]
    got = tbe.cache_attention(q[:, 4:8], Cache(*by_head, c.k_scales, c.v_scales), s["q_offsets"], s["k_offsets"], s["ws"], out=wide[:, 2:6])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool((wide[:, :2] == 7).all()) and bool((wide[:, 6:] == 7).all())
    assert tbe.cache_attention(s["q"], c, s["q_offsets"], s["k_offsets"], s["ws"], stats=False)[1] is None


def test_equals_attention_over_the_values(tbe):
    """tbe_attention over the cache's values read back (exact in fp32 for e4m3, whose scales are powers of two): both are within the same bounds."""
    nq, nk = [1, 5, 40], [700, 90, 400]
    for io in IO:
        s = build(tbe, gen(5), nq, nk, nk, 8, 2, 64, io, E4M3, poison=False)
        k, v = tbe.cache_read(s["cache"], torch.arange(sum(nk), device="cuda"), dtype=io)
        ws = tbe.alloc_attention_workspace(3, sum(nq), sum(nk), 8, 2, 64)
        other = tbe.attention(s["q"], k, v, s["q_offsets"], s["k_offsets"], ws)
        got = compare(tbe, s, nq, nk, "values")
        ref = reference(s["q"], k, v, nq, nk, s["k0"], causal=True, scale=0.125)
        check(other, ref, ("out", "lse"), "attention")
        assert (got[0].double() - other[0].double()).abs().max() <= 2 * ref["~out"].max()


def seen_by(nq, nk, k0, key, causal=True):
    """Rows of q that see row `key` of the cache."""
    a, rows = 0, []
    for n, m, c in zip(nq, nk, k0):
        if c <= key < c + m:
            rows += [a + i for i in range(n) if not causal or key - c <= m - n + i]
        a += n
    return rows


@pytest.mark.parametrize("io", IO)
@pytest.mark.parametrize("code", [E4M3, I8])
@pytest.mark.parametrize("buckets", [0, 16])
def test_what_is_not_finite_reaches_those_that_see_it(tbe, io, code, buckets):
    """A row of the cache made of a head that was not finite, or with a code that is not a number: the queries that see it, and bit for bit no others."""
    for H, K, dim, nq, nk in ((4, 2, 32, [5, 31, 33], [9, 300, 1000]), (2, 2, 128, [6, 1], [300, 270]), (8, 1, 64, [3, 2, 1, 1], [100, 40, 7, 60])):
        g = gen(6)
        s = build(tbe, g, nq, nk, nk, H, K, dim, io, code, buckets=buckets, poison=False)
        clean = run(tbe, s)
        group = H // K
        for n in range(len(nq)):
            for back in (1, 2, min(nk[n], nq[n] + 1), min(nk[n], 200)):
                key, kvh = s["k0"][n] + nk[n] - back, n % K
                for which in ("k_scales", "v_scales") + (("k", "v") if code == E4M3 else ()):
                    t = getattr(s["cache"], which)
                    if which in "kv":
                        t = t.view(torch.uint8)
                        at, bad = (key, kvh, dim // 2 + 1), 0xFF
                    else:
                        at, bad = (kvh, key), math.nan
                    old = t[at].clone()
                    t[at] = bad
                    got = run(tbe, s)
                    t[at] = old
                    hit = torch.zeros(sum(nq), H, dim, dtype=torch.bool, device="cuda")
                    for r in seen_by(nq, nk, s["k0"], key):
                        if which == "v":
                            hit[r, kvh * group:(kvh + 1) * group, dim // 2 + 1] = True
                        else:
                            hit[r, kvh * group:(kvh + 1) * group] = True
                    assert bool(got[0][hit].isnan().all()), (which, n, back)
                    assert torch.equal(got[0][~hit], clean[0][~hit]), (which, n, back)


def test_queries_that_are_not_finite(tbe):
    for io in IO:
        for bad in (math.nan, math.inf):
            nq, nk = [3, 33], [300, 500]
            s = build(tbe, gen(7), nq, nk, nk, 4, 2, 64, io, E4M3, poison=False)
            clean = run(tbe, s)
            s["q"][20, 1, 7] = bad
            got = run(tbe, s)
            hit = torch.zeros_like(s["q"], dtype=torch.bool)
            hit[20, 1] = True
            assert bool(got[0][20, 1].isnan().all()) and torch.equal(got[0][~hit], clean[0][~hit])


def test_hidden_buckets(tbe):
    """A bias of -infinity hides what it falls on, scores and values that are not finite too; a row that sees nothing gets zeros."""
    for io in IO:
        nq, nk = [1, 7], [400, 60]
        s = build(tbe, gen(8), nq, nk, nk, 2, 2, 32, io, E4M3, buckets=8, far=20)
        s["bias"][0, 0] = -math.inf   # the key at the query's own place
        s["bias"][1, :] = -math.inf
        got = run(tbe, s)
        assert bool((got[0][:, 1] == 0).all()) and bool((got[1][1] == -math.inf).all())
        ref = reference(s["q"], values(s["cache"], "k"), values(s["cache"], "v"), nq, nk, s["k0"], causal=True, scale=32 ** -0.5, bias=s["bias"], map_=s["bucket_map"])
        check(got, ref, ("out", "lse"), "hidden")
        s["cache"].k_scales[0, 459] = s["cache"].v_scales[0, 459] = math.nan   # seen by the last query alone, for which it is hidden
        s["cache"].v.view(torch.uint8)[399] = 0x7F
        again = run(tbe, s)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


def test_values_of_very_different_sizes(tbe):
    """Scales from 2^-100 to 2^100 beside each other, in every type of q whose results hold them."""
    for io in (torch.float32, torch.bfloat16):
        g = gen(9)
        nq, nk = [1, 2], [300, 290]
        s = build(tbe, g, nq, nk, nk, 2, 1, 64, io, E4M3, poison=False)
        s["cache"].v_scales.copy_(torch.exp2(torch.randint(-100, 101, s["cache"].v_scales.shape, generator=g, device="cuda").float()))
        compare(tbe, s, nq, nk, "sizes")
    s = build(tbe, gen(10), [1, 2], [300, 290], [300, 290], 2, 1, 64, torch.float16, E4M3, poison=False)
    s["cache"].v_scales.mul_(2.0 ** -12)   # (results near binary16's smallest normal numbers)
    compare(tbe, s, [1, 2], [300, 290], "small")


def test_offsets_that_do_not_fit_are_reported(tbe):
    nq, nk = [1, 2, 1], [300, 40, 500]
    s = build(tbe, gen(11), nq, nk, nk, 2, 2, 32, torch.bfloat16, I8, poison=False)
    good = run(tbe, s)
    torch.cuda.synchronize()
    assert not tbe.poll_index_error()
    for name, at, to in (("k_lengths", 1, 41), ("k_lengths", 0, -1), ("k_offsets", 3, 839), ("k_offsets", 1, 400), ("q_offsets", 1, 4), ("q_offsets", 0, 1), ("k_offsets", 2, -7),
                         ("k_offsets", 1, 2 ** 40)):
        bad = dict(s)
        bad[name] = s[name].clone()
        bad[name][at] = to
        run(tbe, bad)
        torch.cuda.synchronize()
        assert tbe.poll_index_error(), (name, at, to)
    assert torch.equal(run(tbe, s)[0], good[0]) and not tbe.poll_index_error()


def test_no_queries_and_no_keys(tbe):
    s = build(tbe, gen(12), [0, 0], [5, 0], [5, 0], 2, 2, 32, torch.float32, I8)
    assert run(tbe, s)[0].shape == (0, 2, 32)
    s = build(tbe, gen(12), [3, 1], [0, 0], [0, 0], 2, 2, 32, torch.float32, I8)
    out, lse = run(tbe, s)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_on_a_stream_and_in_graphs(tbe):
    """Two graphs on one workspace, replayed in turn with eager calls between them."""
    nq, nk = [1] * 5, [4000, 30, 700, 2000, 900]
    a, b = (build(tbe, gen(13 + i), nq, nk, [n + 5 for n in nk], 8, 2, 64, torch.bfloat16, (E4M3, I8)[i]) for i in range(2))
    b["ws"] = a["ws"]
    want = [run(tbe, s) for s in (a, b)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = run(tbe, a, stream=stream)
    stream.synchronize()
    assert torch.equal(got[0], want[0][0])
    graphs, outs = [], []
    for s in (a, b):
        out = torch.zeros_like(s["q"])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run(tbe, s, out=out, stats=False)
        graphs.append(graph)
        outs.append(out)
    for n in range(3):
        for i, s in enumerate((a, b)):
            outs[i].zero_()
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], run(tbe, s)[0]), (n, i)
        a["k_lengths"].sub_(11)
        b["q"].mul_(1.1)


def test_refusals(tbe):
    from paper_2508_03854_amd import TbeError, binding as B
    s = build(tbe, gen(15), [1, 1], [300, 3000], [300, 3000], 4, 2, 32, torch.float32, E4M3)
    q, c, qo, ko, ws = s["q"], s["cache"], s["q_offsets"], s["k_offsets"], s["ws"]
    for bad, kind in ((lambda: tbe.cache_attention(q[..., :16], c, qo, ko, ws), ValueError), (lambda: tbe.cache_attention(q.double(), c, qo, ko, ws), ValueError),
                      (lambda: tbe.cache_attention(q[0], c, qo, ko, ws), ValueError), (lambda: tbe.cache_attention(q, c, qo, ko[:-1], ws), ValueError),
                      (lambda: tbe.cache_attention(q, c, qo, ko.int(), ws), TypeError), (lambda: tbe.cache_attention(q, c, qo, ko, ws, bias=q[0]), ValueError),
                      (lambda: tbe.cache_attention(q, c, qo, ko, ws, out=q[:1]), ValueError), (lambda: tbe.cache_attention(q.cpu(), c, qo, ko, ws), ValueError)):
        with pytest.raises(kind):
            bad()
    for bad, status in ((lambda: tbe.cache_attention(q[:, :3], c, qo, ko, ws), B.ESHAPE), (lambda: tbe.cache_attention(q, c, qo, ko, None), B.EINVAL),
                        (lambda: tbe.cache_attention(q, c, qo, ko, ws[:256]), B.EWORKSPACE), (lambda: tbe.cache_attention(q, c, qo, ko, ws, scale=math.inf), B.EINVAL),
                        (lambda: tbe.cache_attention_workspace_bytes(1, 1, 1, 1, 1, 24), B.ESHAPE), (lambda: tbe.cache_attention_workspace_bytes(0, 1, 1, 1, 1, 16), B.ESHAPE)):
        with pytest.raises(TbeError) as e:
            bad()
        assert e.value.status == status
    # the cache's sizes and the call's, which the binding cannot make differ
    packed = tbe._pack_attention(q, (c.k.shape[0] - 1, 2, 32), (0,) * 6, qo, ko, None, True, None, None, None)
    assert tbe._lib.tbe_cache_attention(tbe._h, packed, c._args(), B._heads(q.clone(), None, "out"), None, ws.data_ptr(), ws.numel(), 0) == B.ESHAPE
