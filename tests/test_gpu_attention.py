"""Attention over packed sequences, forward, against its definition in 64 bits (tests/attention_reference.py derives the bounds): every
length around a tile's border and none at all, more queries than keys, grouped heads, odd head sizes, both orders, biases by distance,
scales of either sign, caches with room left, offsets of both types, strided operands, values that are not finite; refusals."""
import math

import pytest
import torch

import attention_reference as R

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EDGES = [1, 0, 2, 31, 32, 33, 63, 64, 65, 5, 96, 127, 128, 129, 0, 200, 257, 7]


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def starts(n, dtype=torch.int64):
    return torch.tensor([0] + list(torch.tensor(n).cumsum(0)), dtype=dtype, device="cuda")


def problem(nq, nk, H, K, D, dtype, seed=0, room=None, buckets=0, far=0, causal=True, ids=torch.int64, mul=1.0, bias_dtype=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * seed + 13 * H + D)
    caps = [n + r for n, r in zip(nk, room)] if room else nk

    def normal(*shape, by=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * by).to(dtype)

    Q, C = sum(nq), sum(caps)
    p = {"q": normal(Q, H, D, by=mul), "k": normal(C, K, D, by=mul), "v": normal(C, K, D), "nq": nq, "nk": nk, "caps": caps,
         "k0": [sum(caps[:i]) for i in range(len(caps))], "q_offsets": starts(nq, ids), "k_offsets": starts(caps, ids),
         "k_lengths": torch.tensor(nk, dtype=ids, device="cuda") if room else None, "bias": None, "bucket_map": None, "causal": causal}
    if buckets:
        p["bias"] = (torch.randn(H, buckets, generator=g, device="cuda")).to(bias_dtype or dtype)
        p["bucket_map"] = R.bucket_map(far, buckets, causal)
    return p


def workspace(tbe, p, backward=False):
    ws = tbe.alloc_attention_workspace(len(p["nq"]), p["q"].shape[0], p["k"].shape[0], p["q"].shape[1], p["k"].shape[1], p["q"].shape[2],
                                       buckets=0 if p["bias"] is None else p["bias"].shape[1], backward=backward)
    return ws.fill_(255)


def options(p):
    return {n: p[n] for n in ("k_lengths", "bias", "bucket_map", "causal")}


def run(tbe, p, scale=None, **kw):
    return tbe.attention(p["q"], p["k"], p["v"], p["q_offsets"], p["k_offsets"], workspace(tbe, p), scale=scale, **options(p), **kw)


def refer(p, scale=None, dout=None):
    return R.reference(p["q"], p["k"], p["v"], p["nq"], p["nk"], p["k0"], causal=p["causal"],
                       scale=p["q"].shape[2] ** -0.5 if scale is None else scale, bias=p["bias"], map_=p["bucket_map"], dout=dout)


def agree(tbe, p, what, scale=None):
    got = run(tbe, p, scale)
    R.check(got, refer(p, scale), ("out", "lse"), what)
    again = run(tbe, p, scale)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1]), what
    assert not tbe.poll_index_error(), what


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_around_tiles(tbe, io, causal):
    for D in (32, 64, 128):
        for buckets, far in ((0, 0), (16, 40)):
            few = problem(EDGES, EDGES, 2, 2, D, TYPES[io], causal=causal, buckets=buckets, far=far)           # 68 rows on average
            agree(tbe, few, f"{io} {D} {buckets} long")
            small = EDGES + [3] * 30
            agree(tbe, problem(small, small, 2, 1, D, TYPES[io], causal=causal, buckets=buckets, far=far), f"{io} {D} {buckets} short")


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
def test_queries_behind_a_cache(tbe, io):
    nk = [300, 1, 0, 33, 700, 64, 129, 10, 2, 40]
    for H, K, D in ((4, 4, 32), (8, 2, 64), (6, 2, 40), (5, 1, 128), (36, 1, 64), (8, 8, 96)):
        for nq in ([1] * 10, [1, 1, 1, 0, 3, 1, 0, 2, 1, 1], [40, 1, 7, 33, 64, 2, 129, 3, 2, 100], [200, 1, 7, 33, 300, 64, 129, 3, 2, 100]):
            for causal, buckets, far in ((True, 0, 0), (True, 32, 128), (False, 9, 20)):
                p = problem(nq, nk, H, K, D, TYPES[io], room=[3, 0, 17, 0, 40, 1, 2, 100, 0, 5], buckets=buckets, far=far, causal=causal, ids=torch.int32)
                # what lies in the room is of no concern, whatever it is
                for n, c, m in zip(p["k0"], p["caps"], p["nk"]):
                    p["k"][n + m:n + c], p["v"][n + m:n + c] = float("nan"), float("inf")
                agree(tbe, p, f"{io} {H}/{K}x{D} {nq[:3]} {causal} {buckets}")


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
def test_long_keys_in_parts(tbe, io):
    """Few wavefronts, many keys: the parts of the keys are joined, some of them empty, some hidden by the order."""
    for H, K, D, nq, nk in ((1, 1, 32, [1], [5000]), (4, 1, 64, [1, 1], [9000, 3]), (2, 2, 128, [20, 1, 31], [3000, 2600, 10]), (8, 8, 64, [3], [777]),
                            (16, 2, 128, [1, 1, 1], [4097, 1, 2048]), (1, 1, 8, [60], [2500])):
        for causal, buckets in ((True, 0), (True, 32), (False, 0)):
            p = problem(nq, nk, H, K, D, TYPES[io], buckets=buckets, far=128, causal=causal)
            agree(tbe, p, f"{io} {H}/{K}x{D} {nk} {causal} {buckets}")


@pytest.mark.parametrize("io,dims", [("f32", (4, 12, 20, 36, 64, 100, 124)), ("f16", (8, 16, 24, 40, 72, 80, 120)), ("bf16", (8, 16, 56, 88, 104, 112))])
def test_head_sizes(tbe, io, dims):
    for D in dims:
        for nq in ([70, 1, 130], [1, 1, 1]):
            agree(tbe, problem(nq, [70, 55, 130], 3, 3, D, TYPES[io], buckets=8, far=12), f"{io} {D} {nq}")


@pytest.mark.parametrize("far", [0, 1, 31, 63, 64, 500, 1024])
def test_bias_by_distance(tbe, far):
    for io, bias_io in (("f32", "f32"), ("bf16", "f32"), ("f16", "f16"), ("f32", "bf16")):
        for causal in (True, False):
            for H, K, nq, nk in ((2, 1, [300, 150], [300, 150]), (4, 1, [1, 1, 2], [300, 1300, 40]), (3, 3, [40, 20], [400, 700])):
                p = problem(nq, nk, H, K, 32, TYPES[io], buckets=13, far=far, causal=causal, bias_dtype=TYPES[bias_io])
                agree(tbe, p, f"{io} {bias_io} {causal} {nq}")


def test_bias_that_hides(tbe):
    """A bucket of -infinity hides its keys, rows of hidden keys alone are empty; a bucket of the type's lowest value hides nothing from rows
    that have nothing else."""
    for io in ("f32", "bf16"):
        for nq in ([300], [1, 1]):
            p = problem(nq, [300] * len(nq), 2, 1, 64, TYPES[io], buckets=8, far=200)
            p["bias"][0, :6] = -math.inf
            p["bias"][1, :] = -math.inf
            got = run(tbe, p)
            R.check(got, refer(p), ("out", "lse"), io)
            assert bool((got[0][:, 1] == 0).all()) and bool((got[1][1] == -math.inf).all())
            # with all buckets at the lowest value the scores vanish in it: every visible key counts the same
            p["bias"][:] = torch.finfo(TYPES[io]).min
            out, _ = run(tbe, p)
            at, c0 = 0, 0
            for n, m in zip(p["nq"], p["nk"]):
                for i in (0, n // 2, n - 1):
                    mean = p["v"][c0:c0 + m - n + i + 1, 0].double().mean(0)
                    assert (out[at + i].double() - mean).abs().max() <= (m + 24) * R.U * 6 + R.T[TYPES[io]] * 12
                at, c0 = at + n, c0 + m
    p = problem([40], [40], 1, 1, 32, torch.float32, buckets=4, far=5)
    p["bias"][0, 0] = math.inf          # infinity minus infinity: the formula's NaN, for every row (distance 0 is seen by all)
    assert bool(torch.isnan(run(tbe, p)[0]).all())


@pytest.mark.parametrize("scale", [-0.7, 0.0, 3.0, 1e-20])
def test_scales(tbe, scale):
    for io in ("f32", "f16"):
        for nq, nk in (([130, 20], [130, 20]), ([1, 3], [90, 33])):
            for buckets in (0, 8):
                agree(tbe, problem(nq, nk, 2, 1, 64, TYPES[io], buckets=buckets, far=9), f"{io} {scale} {nq} {buckets}", scale)


def test_large_scores_and_late_maxima(tbe):
    """Scores of a few hundred that grow along the keys: the running maximum moves in nearly every tile."""
    for nq, nk in (([256], [256]), ([1], [3000])):
        p = problem(nq, nk, 1, 1, 32, torch.float32)
        p["q"][:], p["k"][:] = 1.0, 0.0
        p["k"][:, 0, 0] = torch.arange(nk[0], device="cuda") * 0.37
        agree(tbe, p, f"{nk} up", 1.0)
        p["k"][:, 0, 0] = torch.arange(nk[0], device="cuda") * -0.37
        agree(tbe, p, f"{nk} down", 1.0)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_strided_operands(tbe, io):
    """q, k and v as column blocks of one matrix, and with the heads outermost; the result between other columns that stay as they are."""
    n = [65, 1, 200, 31]
    p = problem(n, n, 4, 2, 32, TYPES[io], buckets=8, far=30)
    ref = run(tbe, p)
    one = torch.cat([p["q"].reshape(-1, 128), p["k"].reshape(-1, 64), p["v"].reshape(-1, 64)], 1)
    s = dict(p, q=one[:, :128].view(-1, 4, 32), k=one[:, 128:192].view(-1, 2, 32), v=one[:, 192:].view(-1, 2, 32))
    buf = torch.full((sum(n), 4, 64), 7.0, dtype=TYPES[io], device="cuda")
    lse = torch.empty(4, sum(n), device="cuda")
    run(tbe, s, out=buf[:, :, 16:48], lse=lse)
    assert torch.equal(buf[:, :, 16:48], ref[0]) and torch.equal(lse, ref[1]) and bool((buf[:, :, :16] == 7).all()) and bool((buf[:, :, 48:] == 7).all())
    s = {**p, **{m: p[m].transpose(0, 1).contiguous().transpose(0, 1) for m in "qkv"}}
    out = torch.empty(4, sum(n), 32, dtype=TYPES[io], device="cuda").transpose(0, 1)
    assert torch.equal(run(tbe, s, out=out, stats=False)[0], ref[0])
    # one key row for all of them: a stride of zero
    s = dict(p, k=p["k"][:1].expand(sum(n), 2, 32), v=p["v"][:1].expand(sum(n), 2, 32))
    got = run(tbe, s)[0]
    assert (got.double() - p["v"][0].repeat_interleave(2, 0).double()).abs().max() <= (R.T[TYPES[io]] * 2 + 300 * R.U) * 5


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite_reach_only_who_sees_them(tbe, io):
    for D in (32, 64, 128):
        for nq, nk in (([200, 70], [200, 70]), ([30, 20], [150, 20]), ([20] * 4, [20] * 4)):
            p = problem(nq, nk, 2, 1, D, TYPES[io])
            clean = run(tbe, p)[0]
            at = [(0, min(nk[0] - 1, nk[0] - nq[0] + 11)), (1, 13)]         # (sequence, key)
            p["v"][p["k0"][0] + at[0][1], 0, 3] = math.inf
            p["v"][p["k0"][1] + at[1][1], 0, 1] = float("nan")
            got = run(tbe, p)[0]
            expect, a = clean.clone(), 0
            for s, (n, m) in enumerate(zip(nq, nk)):
                for q, key, col, x in ((0, at[0][1], 3, math.inf), (1, at[1][1], 1, float("nan"))):
                    if q == s:
                        expect[a + max(0, key - (m - n)):a + n, :, col] = x
                a += n
            seen = torch.isfinite(expect)
            assert torch.equal(torch.isnan(got), torch.isnan(expect)) and torch.equal(got == math.inf, expect == math.inf), (D, nq)
            assert (got[seen].double() - clean[seen].double()).abs().max() <= 4 * (R.T[TYPES[io]] + 300 * R.U) * clean[seen].abs().max().double()
            # a key that is not finite reaches the queries that see it, and no other
            p = problem(nq, nk, 2, 1, D, TYPES[io])
            p["k"][p["k0"][0] + at[0][1], 0, 2] = float("nan")
            got = run(tbe, p)[0]
            row = max(0, at[0][1] - (nk[0] - nq[0]))
            assert bool(torch.isnan(got[row:nq[0]]).all()) and torch.equal(got[:row], clean[:row]) and torch.equal(got[nq[0]:], clean[nq[0]:])


def test_offsets_that_do_not_fit_are_reported(tbe):
    n = [40, 30, 20]
    p = problem(n, n, 2, 1, 32, torch.float32)
    ref = run(tbe, p)[0]
    for what, where, values in (("descending", "q_offsets", [0, 40, 30, 90]), ("behind the end", "q_offsets", [0, 40, 70, 95]),
                                ("short", "q_offsets", [0, 40, 70, 80]), ("not from 0", "k_offsets", [1, 40, 70, 90]),
                                ("keys descending", "k_offsets", [0, 40, 35, 90]), ("far out", "k_offsets", [0, 40, 1 << 40, 90]),
                                ("negative", "k_offsets", [0, -5, 70, 90])):
        s = dict(p)
        s[where] = torch.tensor(values, dtype=torch.int64, device="cuda")
        buf = torch.full((90, 2, 32), 7.0, device="cuda")
        run(tbe, s, out=buf)
        assert tbe.poll_index_error(), what
        assert torch.isfinite(buf).all(), what
    s = dict(p, k_lengths=torch.tensor([40, 31, 20], device="cuda"))
    buf = torch.full((90, 2, 32), 7.0, device="cuda")
    run(tbe, s, out=buf)
    assert tbe.poll_index_error() and torch.equal(buf[:40], ref[:40]) and bool((buf[40:70] == 7).all()) and torch.equal(buf[70:], ref[70:])
    # a bucket outside the table: no bias, reported
    s = problem(n, n, 2, 1, 32, torch.float32, buckets=4, far=3)
    s["bucket_map"][:] = 4
    got = run(tbe, s)[0]
    assert tbe.poll_index_error()
    assert (got - run(tbe, dict(s, bias=None, bucket_map=None))[0]).abs().max() < 1e-5


def test_nothing_to_do(tbe):
    for nq, nk in (([0, 0], [5, 0]), ([3, 2], [0, 0]), ([0], [0])):
        p = problem(nq, nk, 2, 2, 32, torch.float32)
        out, lse = run(tbe, p)
        assert out.shape == p["q"].shape and bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_many_sequences(tbe):
    """More sequences than one search step tells apart, most of them empty or of one row."""
    n = [(i * 7919) % 4 if i % 97 else 60 for i in range(5000)]
    p = problem(n, n, 1, 1, 8, torch.float32, ids=torch.int32)
    out, _ = run(tbe, p)


    # a handful of places all over, one sequence at a time
    for i in list(range(0, 5000, 173)) + [4999, 97 * 51]:
        a, m = p["k0"][i], n[i]
        if m:
            part = R.reference(p["q"][a:a + m], p["k"][a:a + m], p["v"][a:a + m], [m], [m], [0], causal=True, scale=8 ** -0.5)
            R.check((out[a:a + m],), part, ("out",), str(i))



def test_rows_beyond_four_gigabytes(tbe):
    """A cache whose rows lie so far apart that byte offsets pass 2^32: the last sequence's keys are found."""
    wide = torch.zeros(70_000, 16 * 1024 * 2, dtype=torch.bfloat16, device="cuda")          # 4.6 GB
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    wide[-300:, :64] = torch.randn(300, 64, generator=g, device="cuda").to(torch.bfloat16)
    k, v = wide[:, :32].view(-1, 1, 32), wide[:, 32:64].view(-1, 1, 32)
    q = torch.randn(2, 1, 32, generator=g, device="cuda").to(torch.bfloat16)
    off, qo = torch.tensor([0, 69_700, 70_000], device="cuda"), torch.tensor([0, 1, 2], device="cuda")
    ws = tbe.alloc_attention_workspace(2, 2, 70_000, 1, 1, 32)
    out, lse = tbe.attention(q, k, v, qo, off, ws)
    ref = R.reference(q[1:], k[-300:], v[-300:], [1], [300], [0], causal=True, scale=32 ** -0.5)
    R.check((out[1:], lse[:, 1:]), ref, ("out", "lse"), "last")
    assert bool((out[0] == 0).all())


def test_streams_graphs_and_timing(tbe):
    n = [100, 3, 260, 64]
    cases = [problem(n, n, 4, 2, 64, torch.bfloat16, buckets=8, far=50), problem([1, 1], [4000, 2500], 4, 2, 64, torch.bfloat16)]
    refs = [run(tbe, p) for p in cases]
    spaces = [workspace(tbe, p) for p in cases]
    got = [(torch.empty_like(o), torch.empty_like(m)) for o, m in refs]
    torch.cuda.synchronize()

    def all_(stream=None):
        for p, ws, (o, m) in zip(cases, spaces, got):
            tbe.attention(p["q"], p["k"], p["v"], p["q_offsets"], p["k_offsets"], ws, out=o, lse=m, stream=stream, **options(p))

    s = torch.cuda.Stream()
    all_(s)
    s.synchronize()
    assert all(torch.equal(a, b) for r, g in zip(refs, got) for a, b in zip(r, g))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_()
    for _ in range(3):
        for o, m in got:
            o.zero_(), m.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for r, g in zip(refs, got) for a, b in zip(r, g))
    tbe.timing_enable(True)
    all_()
    names = [x for x, _ in tbe.timing_read()]
    tbe.timing_enable(False)
    assert names == ["attention", "attention", "attention_join"]


def test_refusals(tbe):
    from paper_2508_03854_amd import binding
    p = problem([5, 6], [5, 6], 4, 2, 32, torch.float32, buckets=4, far=3)

    def status(scale=None, **kw):
        s = {**p, **kw}
        with pytest.raises(binding.TbeError) as e:
            tbe.attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], s.get("ws", workspace(tbe, p)), scale=scale, **options(s))
        return e.value.status

    for scale in (math.nan, math.inf):
        assert status(scale) == binding.EINVAL
    z = torch.zeros
    assert status(q=z(11, 3, 32, device="cuda"), bias=z(3, 4, device="cuda")) == binding.ESHAPE              # 3 heads on 2
    assert status(q=z(11, 4, 132, device="cuda"), k=z(11, 2, 132, device="cuda"), v=z(11, 2, 132, device="cuda")) == binding.ESHAPE
    assert status(q=z(11, 4, 6, device="cuda"), k=z(11, 2, 6, device="cuda"), v=z(11, 2, 6, device="cuda")) == binding.ESHAPE
    assert status(bucket_map=z(2051, dtype=torch.int32, device="cuda")) == binding.ESHAPE
    assert status(q=z(11 * 4 * 32 + 1, device="cuda")[1:].view(11, 4, 32)) == binding.EINVAL                 # not on 16 bytes
    assert status(q=z(11, 4, 34, device="cuda")[:, :, :32]) == binding.EINVAL                                # nor its heads
    assert status(q_offsets=z(1, dtype=torch.int64, device="cuda"), k_offsets=z(1, dtype=torch.int64, device="cuda")) == binding.ESHAPE
    one = problem([1], [5000], 4, 2, 32, torch.float32)
    need = tbe.attention_workspace_bytes(1, 1, 5000, 4, 2, 32)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for bad, why in ((None, binding.EINVAL), (ws[:need // 4], binding.EWORKSPACE), (ws[1:], binding.EINVAL)):
        with pytest.raises(binding.TbeError) as e:
            tbe.attention(one["q"], one["k"], one["v"], one["q_offsets"], one["k_offsets"], bad)
        assert e.value.status == why
    q, k, v, qo, ko = (p[n] for n in ("q", "k", "v", "q_offsets", "k_offsets"))
    for err, bad in ((ValueError, lambda: tbe.attention(q[0], k, v, qo, ko, None)), (ValueError, lambda: tbe.attention(q, k, v[:-1], qo, ko, None)),
                     (ValueError, lambda: tbe.attention(q, k.half(), v, qo, ko, None)), (ValueError, lambda: tbe.attention(q.cpu(), k, v, qo, ko, None)),
                     (ValueError, lambda: tbe.attention(q, k, v, qo, ko[:-1], None)), (TypeError, lambda: tbe.attention(q, k, v, qo.int(), ko, None)),
                     (ValueError, lambda: tbe.attention(q, k, v, qo, ko, None, bias=p["bias"])), (TypeError, lambda: tbe.attention(q.double(), k, v, qo, ko, None)),
                     (TypeError, lambda: tbe.attention(q, k, v, qo, ko, None, bias=p["bias"], bucket_map=p["bucket_map"].long())),
                     (ValueError, lambda: tbe.attention(q, k, v, qo, ko, None, out=q[:5])),
                     (ValueError, lambda: tbe.attention(q.transpose(1, 2), k, v, qo, ko, None))):
        with pytest.raises(err):
            bad()
    L = binding.load_library()
    assert L.tbe_attention(tbe._h, None, binding.Rows(), None, None, 0, None) == binding.EINVAL
    a = binding.AttentionArgs(sequences=1, heads=1, kv_heads=1, head_dim=8, dtype=5)
    import ctypes
    assert L.tbe_attention(tbe._h, ctypes.addressof(a), binding.Rows(), None, None, 0, None) == binding.EDTYPE
