"""Gradients of attention over packed sequences against the formula in 64 bits (tests/attention_reference.py derives the bounds) and
against differences: every length around a tile's border and none at all, grouped heads in parts, odd head sizes, both orders, the
bias's gradient, scales of either sign, caches with room, strided operands; refusals."""
import math

import pytest
import torch

import attention_reference as R
from test_gpu_attention import EDGES, TYPES, options, problem, refer, run, workspace

pytestmark = pytest.mark.gpu
NAMES = ("dq", "dk", "dv", "dbias")


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def upstream(p, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(77 + seed)
    return torch.randn(p["q"].shape, generator=g, device="cuda").to(p["q"].dtype)


def back(tbe, p, dout, fwd, scale=None, **kw):
    ws = kw.pop("ws", None)
    return tbe.attention_backward(dout, p["q"], p["k"], p["v"], fwd[0], fwd[1], p["q_offsets"], p["k_offsets"],
                                  workspace(tbe, p, True) if ws is None else ws, scale=scale, **options(p), **kw)


def agree(tbe, p, what, scale=None):
    dout = upstream(p)
    fwd = run(tbe, p, scale)
    got = back(tbe, p, dout, fwd, scale)
    n = 4 if p["bias"] is not None else 3
    R.check(got[:n], refer(p, scale, dout), NAMES[:n], what)
    again = back(tbe, p, dout, fwd, scale)
    assert all(torch.equal(a, b) for a, b in zip(got[:n], again[:n])), what
    assert not tbe.poll_index_error(), what


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_around_tiles(tbe, io, causal):
    for D in (32, 64, 128):
        for buckets, far in ((0, 0), (16, 40)):
            agree(tbe, problem(EDGES, EDGES, 2, 2, D, TYPES[io], causal=causal, buckets=buckets, far=far), f"{io} {D} {buckets} long")
            small = EDGES + [3] * 30
            agree(tbe, problem(small, small, 2, 1, D, TYPES[io], causal=causal, buckets=buckets, far=far), f"{io} {D} {buckets} short")


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
def test_other_numbers_of_queries_and_keys(tbe, io):
    nk = [300, 1, 0, 33, 400, 64, 129, 10, 2, 40]
    for H, K, D in ((4, 4, 32), (8, 2, 64), (6, 1, 40), (5, 1, 128), (12, 2, 64)):
        for nq in ([1, 1, 1, 0, 3, 1, 0, 2, 1, 1], [40, 1, 7, 33, 64, 2, 129, 3, 2, 100], [200, 1, 7, 33, 300, 64, 129, 3, 2, 100]):
            for causal, buckets, far in ((True, 32, 128), (False, 9, 20), (True, 0, 0)):
                p = problem(nq, nk, H, K, D, TYPES[io], room=[3, 0, 17, 0, 40, 1, 2, 100, 0, 5], buckets=buckets, far=far, causal=causal, ids=torch.int32)
                for n, c, m in zip(p["k0"], p["caps"], p["nk"]):
                    p["k"][n + m:n + c], p["v"][n + m:n + c] = float("nan"), float("inf")
                agree(tbe, p, f"{io} {H}/{K}x{D} {nq[:3]} {causal} {buckets}")


@pytest.mark.parametrize("io,dims", [("f32", (4, 12, 36, 100)), ("f16", (8, 24, 72, 120)), ("bf16", (16, 56, 96, 112))])
def test_head_sizes(tbe, io, dims):
    for D in dims:
        for n in ([70, 1, 130], [9, 30, 20]):
            agree(tbe, problem(n, n, 3, 3, D, TYPES[io], buckets=8, far=12), f"{io} {D} {n}")


@pytest.mark.parametrize("far", [0, 1, 31, 64, 200, 1024])
def test_bias_by_distance(tbe, far):
    for io, bias_io in (("f32", "f32"), ("bf16", "f32"), ("f16", "f16"), ("f32", "bf16")):
        for causal in (True, False):
            for H, K, D, nq, nk in ((2, 1, 32, [300, 150], [300, 150]), (2, 2, 128, [40, 20], [400, 700]), (4, 1, 64, [20, 31, 5], [20, 31, 50])):
                agree(tbe, problem(nq, nk, H, K, D, TYPES[io], buckets=13, far=far, causal=causal, bias_dtype=TYPES[bias_io]), f"{io} {bias_io} {causal} {nq}")


def test_many_buckets_and_few(tbe):
    for buckets in (1, 3, 200, 1024):
        for n in ([150, 90], [20, 12, 9]):
            agree(tbe, problem(n, n, 2, 2, 32, torch.float32, buckets=buckets, far=600), f"{buckets} {n}")


def test_hidden_buckets_have_no_gradient(tbe):
    for n in ([300], [30, 20]):
        p = problem(n, n, 2, 1, 64, torch.float32, buckets=8, far=200)
        p["bias"][0, :3] = -math.inf
        p["bias"][1, :] = -math.inf
        dout, fwd = upstream(p), run(tbe, p)
        got = back(tbe, p, dout, fwd)
        assert all(bool(torch.isfinite(t).all()) for t in got)
        assert bool((got[0][:, 1] == 0).all()) and bool((got[3][1] == 0).all()) and bool((got[3][0, :3] == 0).all())


@pytest.mark.parametrize("scale", [-0.7, 0.0, 2.0])
def test_scales(tbe, scale):
    for io in ("f32", "f16"):
        for n in ([130, 20], [30, 3]):
            for buckets in (0, 8):
                agree(tbe, problem(n, n, 2, 1, 64, TYPES[io], buckets=buckets, far=9), f"{io} {scale} {n} {buckets}", scale)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_strided_operands(tbe, io):
    """All operands and gradients as column blocks of wider matrices; what lies between stays as it is."""
    for n in ([65, 1, 200, 31], [20, 7, 30]):
        p = problem(n, n, 4, 2, 32, TYPES[io], buckets=8, far=30)
        dout, fwd = upstream(p), run(tbe, p)
        ref = back(tbe, p, dout, fwd)
        N = sum(n)
        one = torch.cat([p["q"].reshape(N, 128), p["k"].reshape(N, 64), p["v"].reshape(N, 64)], 1)
        s = dict(p, q=one[:, :128].view(N, 4, 32), k=one[:, 128:192].view(N, 2, 32), v=one[:, 192:].view(N, 2, 32))
        buf = torch.full((N, 288), 7.0, dtype=TYPES[io], device="cuda")
        blocks = [buf[:, 16:144].view(N, 4, 32), buf[:, 144:208].view(N, 2, 32), buf[:, 208:272].view(N, 2, 32)]
        back(tbe, s, dout.transpose(0, 1).contiguous().transpose(0, 1), fwd, grad_q=blocks[0], grad_k=blocks[1], grad_v=blocks[2])
        assert all(torch.equal(a, b) for a, b in zip(blocks, ref)) and bool((buf[:, :16] == 7).all()) and bool((buf[:, 272:] == 7).all())


def test_against_differences(tbe):
    """sum(out * dout) in 64 bits at x +- d e: the central difference is off by d^2 / 6 of the third derivative, below 1e-6 here; the fp32
    kernels are held to 2e-5 of the largest gradient."""
    p = problem([5, 3], [5, 6], 2, 1, 4, torch.float32, buckets=4, far=3)
    dout, fwd = upstream(p), run(tbe, p)
    got = back(tbe, p, dout, fwd)

    def loss(q, k, v, b):
        r = R.reference(q, k, v, p["nq"], p["nk"], p["k0"], causal=True, scale=0.5, bias=b, map_=p["bucket_map"])
        return (r["out"] * dout.double()).sum().item()

    at = [p["q"].double(), p["k"].double(), p["v"].double(), p["bias"].double()]
    R.T[torch.float64], R.TINY[torch.float64] = 0.0, 0.0
    for k, grad in enumerate(got):
        num = torch.zeros(at[k].numel(), dtype=torch.float64)
        for e in range(num.numel()):
            side = []
            for d in (1e-4, -1e-4):
                x = [t.clone() for t in at]
                x[k].view(-1)[e] += d
                side.append(loss(*x))
            num[e] = (side[0] - side[1]) / 2e-4
        assert (num - grad.double().cpu().view(-1)).abs().max() <= 2e-5 * max(1.0, num.abs().max().item()), NAMES[k]


def test_nothing_to_do(tbe):
    for nq, nk in (([0, 0], [5, 0]), ([3, 2], [0, 0]), ([0], [0])):
        p = problem(nq, nk, 2, 2, 32, torch.float32, buckets=4, far=2)
        dout, fwd = upstream(p), run(tbe, p)
        assert all(bool((t == 0).all()) for t in back(tbe, p, dout, fwd))


def test_what_is_not_finite_stays_in_its_sequence(tbe):
    n = [40, 100, 33]
    for io in ("f32", "bf16"):
        p = problem(n, n, 2, 1, 64, TYPES[io])
        dout, fwd = upstream(p), run(tbe, p)
        clean = back(tbe, p, dout, fwd)
        dout[60, 1, 3] = math.nan
        got = back(tbe, p, dout, fwd)
        for a, b in zip(got[:3], clean[:3]):
            assert torch.equal(a[:40], b[:40]) and torch.equal(a[140:], b[140:])
        assert bool(torch.isnan(got[0][60, 1]).all())


def test_offsets_that_do_not_fit_are_reported(tbe):
    n = [40, 30, 20]
    p = problem(n, n, 2, 1, 32, torch.float32, buckets=4, far=3)
    dout, fwd = upstream(p), run(tbe, p)
    for where, values in (("q_offsets", [0, 40, 30, 90]), ("q_offsets", [0, 40, 70, 95]), ("k_offsets", [1, 40, 70, 90]),
                          ("k_offsets", [0, 40, 35, 90]), ("k_offsets", [0, 40, 1 << 40, 90]), ("k_offsets", [0, -5, 70, 90])):
        s = dict(p)
        s[where] = torch.tensor(values, dtype=torch.int64, device="cuda")
        back(tbe, s, dout, fwd)
        assert tbe.poll_index_error(), values


def test_streams_graphs_and_timing(tbe):
    n = [100, 3, 260, 64]
    cases = [problem(n, n, 4, 2, 64, torch.bfloat16, buckets=8, far=50), problem([9, 20], [9, 20], 2, 2, 32, torch.bfloat16)]
    ups, fwds = [upstream(p) for p in cases], [run(tbe, p) for p in cases]
    refs = [back(tbe, p, u, f) for p, u, f in zip(cases, ups, fwds)]
    spaces = [workspace(tbe, p, True) for p in cases]
    got = [[None if t is None else torch.empty_like(t) for t in r] for r in refs]
    torch.cuda.synchronize()

    def all_(stream=None):
        for p, u, f, ws, g in zip(cases, ups, fwds, spaces, got):
            back(tbe, p, u, f, ws=ws, grad_q=g[0], grad_k=g[1], grad_v=g[2], grad_bias=g[3], stream=stream)

    def same():
        return all(torch.equal(a, b) for r, g in zip(refs, got) for a, b in zip(r, g) if a is not None)

    s = torch.cuda.Stream()
    all_(s)
    s.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_()
    for _ in range(3):
        for g in got:
            for t in g:
                if t is not None:
                    t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same()
    tbe.timing_enable(True)
    all_()
    names = [x for x, _ in tbe.timing_read()]
    tbe.timing_enable(False)
    assert names[:3] == ["attention_dq", "attention_dbias", "attention_dkv"] and "attention_dkv" in names[3:]


def test_refusals(tbe):
    from paper_2508_03854_amd import binding
    n = [5, 60]
    p = problem(n, n, 4, 2, 32, torch.float32, buckets=4, far=3)
    dout, fwd = upstream(p), run(tbe, p)
    ws = workspace(tbe, p, True)

    def status(**kw):
        with pytest.raises(binding.TbeError) as e:
            back(tbe, p, dout, fwd, **kw)
        return e.value.status

    assert status(ws=ws[:256]) == binding.EWORKSPACE and status(ws=ws[1:]) == binding.EINVAL
    with pytest.raises(binding.TbeError) as e:
        tbe.attention_backward(dout, p["q"], p["k"], p["v"], fwd[0], fwd[1], p["q_offsets"], p["k_offsets"], None, **options(p))
    assert e.value.status == binding.EINVAL
    assert status(scale=math.nan) == binding.EINVAL
    assert status(grad_k=torch.empty(65 * 64 + 1, device="cuda")[1:].view(65, 2, 32)) == binding.EINVAL
    assert status(grad_q=torch.empty(1, 4, 32, device="cuda").expand(65, 4, 32)) == binding.EINVAL
    for err, kw in ((ValueError, {"grad_q": torch.empty(64, 4, 32, device="cuda")}), (ValueError, {"grad_v": torch.empty(65, 2, 32, dtype=torch.half, device="cuda")}),
                    (TypeError, {"grad_bias": torch.empty(4, 4, dtype=torch.half, device="cuda")}), (ValueError, {"grad_bias": torch.empty(4, 5, device="cuda")})):
        with pytest.raises(err):
            back(tbe, p, dout, fwd, **kw)
    with pytest.raises(ValueError):
        back(tbe, dict(p, bias=None, bucket_map=None), dout, fwd, grad_bias=torch.empty(4, 4, device="cuda"))
