"""Rotation, attention and caches of one byte an element as they are used together: gradients of the example's chain with rotated heads against
64-bit automatic differentiation; prompts and single events served from a cache against the whole sequences in 64 bits; the whole step in a graph."""
import math
import os
import sys

import pytest
import torch

from attention_reference import check, reference

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E4M3, I8 = torch.float8_e4m3fn, torch.int8
U = 2.0 ** -24


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import event_encoder
    return event_encoder


def turn64(x, w, places, freq):
    """[rows, heads, dim] normed and rotated in 64 bits, halves against each other."""
    x = x / (x.square().mean(2, keepdim=True) + 1e-6).sqrt() * w
    t = (places.double()[:, None] * freq)[:, None]
    a, b = x.chunk(2, 2)
    return torch.cat((a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()), 2)


def test_gradients_of_the_chain_with_rotated_heads(example):
    """fp32: each operator within a few hundred units of 2^-24 of its operands (see their own tests); the norm of heads amplifies what comes before it by the
    heads' reciprocal norms, at most 4 here; four in turn within 2e-4 of the largest gradient."""
    enc = example.EventEncoder(50, seed=3, rotary=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    for p in (enc.weight, enc.norm_bias, enc.bias, enc.q_weight, enc.k_weight):
        p += 0.3 * torch.randn(p.shape, generator=g, device="cuda")
    n, offsets = [7, 1, 40, 13], torch.tensor([0, 7, 8, 48, 61], device="cuda")
    ids = torch.randint(0, 50, (61,), generator=g, device="cuda")
    f = enc.forward(ids, offsets)
    dout = torch.randn(61, enc.heads, enc.dim, generator=g, device="cuda")
    got = enc.gradients(f, dout, offsets)
    assert len(got) == 6
    leaves = [t.double().detach().requires_grad_() for t in (enc.tables.view(50, -1)[ids], enc.weight, enc.norm_bias, enc.bias, enc.q_weight, enc.k_weight)]
    x, w, b, table, qw, kw = leaves
    y = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt() * w + b
    q, k, v = y.view(-1, 3 * enc.heads, enc.dim).split(enc.heads, 1)
    assert 1 / q.square().mean(2).sqrt().min() < 4 and 1 / k.square().mean(2).sqrt().min() < 4
    places = torch.cat([torch.arange(m, device="cuda") for m in n])
    q, k = turn64(q, qw, places, enc.frequencies), turn64(k, kw, places, enc.frequencies)
    outs, far = [], enc.bucket_map.numel() // 2
    for i, m in enumerate(n):
        s = slice(int(offsets[i]), int(offsets[i + 1]))
        d = torch.arange(m, device="cuda")[:, None] - torch.arange(m, device="cuda")
        score = torch.einsum("ihd,jhd->hij", q[s], k[s]) * enc.dim ** -0.5 + table[:, enc.bucket_map.long()[d.clamp(-far, far) + far]]
        outs.append(torch.einsum("hij,jhd->ihd", score.masked_fill(d < 0, -math.inf).softmax(2), v[s]))
    out = torch.cat(outs)
    assert (f["out"].double() - out).abs().max() <= 2e-4 * out.abs().max()
    out.backward(dout.double())
    for a, leaf in zip(got, leaves):
        assert (a.double() - leaf.grad).abs().max() <= 2e-4 * leaf.grad.abs().max()


@pytest.mark.parametrize("args", [["--rotary"], ["--rotary", "--cache", "e4m3"], ["--cache", "i8", "--io", "bf16"], ["--rotary", "--cache", "i8", "--io", "f16"]])
def test_the_example_runs(example, args):
    losses, worst = example.main(["--steps", "5", "--users", "32", "--ids", "60", *args])
    assert all(math.isfinite(x) for x in losses) and math.isfinite(worst)


@pytest.mark.parametrize("io", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("code", [E4M3, I8])
def test_a_prompt_and_single_events_through_the_cache(example, io, code):
    """q, k and v of whole histories; a prompt of each goes into the cache at once, the others one by one; every answer is that of the definition over
    what the cache's bytes stand for, and those are within half a step of the rotated keys and the values."""
    from paper_2508_03854_amd import TBE, rotary_frequencies
    tbe, H, K, dim = TBE([16], [8]), 4, 2, 64
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    prompts, steps, room = [37, 1, 300, 64], 6, 320
    N, freq = len(prompts), rotary_frequencies(dim)
    w = [torch.rand(dim, generator=g, device="cuda") + 0.5 for _ in range(2)]
    rows = [torch.randn(n + steps, H + 2 * K, dim, generator=g, device="cuda").to(io) for n in prompts]
    cache, starts = tbe.alloc_cache(N * room, K, dim, code), torch.arange(N + 1, device="cuda") * room
    for t in (cache.k, cache.v):
        t.view(torch.uint8).fill_(0x7F)
    lengths = torch.zeros(N, dtype=torch.int64, device="cuda")

    def step(new, places, nq, causal=True):
        x = torch.cat(new)
        q, k, v = x.split((H, K, K), 1)
        q, k = tbe.rotate_heads(q, k, places, freq, norm=True, q_weight=w[0], k_weight=w[1])
        seq = torch.repeat_interleave(torch.arange(N, device="cuda"), torch.tensor(nq, device="cuda"))
        tbe.cache_write(cache, k, v, starts[seq] + places)
        lengths.copy_(places[torch.tensor(nq, device="cuda").cumsum(0) - 1] + 1)
        qo = torch.tensor([sum(nq[:i]) for i in range(N + 1)], device="cuda")
        ws = tbe.alloc_cache_attention_workspace(N, len(x), N * room, H, K, dim)
        got = tbe.cache_attention(q, cache, qo, starts, ws, k_lengths=lengths)
        values = [c.float().double() * s.t().double()[..., None] for c, s in ((cache.k, cache.k_scales), (cache.v, cache.v_scales))]
        ref = reference(q, *values, nq, lengths.tolist(), starts[:-1].tolist(), causal=True, scale=dim ** -0.5)
        check(got, ref, ("out", "lse"), "step")

    step([r[:n] for r, n in zip(rows, prompts)], torch.cat([torch.arange(n, device="cuda") for n in prompts]), prompts)
    for t in range(steps):
        step([r[n + t:n + t + 1] for r, n in zip(rows, prompts)], torch.tensor([n + t for n in prompts], device="cuda"), [1] * N)
    # half a step: of a code's 3 fraction bits (e4m3, 2^-4 of it, 2^-10 of the scale below its normal numbers), of a whole number; before it, the keys' rounding
    half = {torch.float32: 40 * U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[io]
    for n, (r, m) in enumerate(zip(rows, prompts)):
        at = torch.arange(n * room, n * room + m + steps, device="cuda")
        got = tbe.cache_read(cache, at)
        k = turn64(r[:, H:H + K].double(), w[1].double(), torch.arange(m + steps, device="cuda"), freq)
        for x, y, s, before in ((got[0], k, cache.k_scales, half), (got[1], r[:, H + K:].double(), cache.v_scales, 0.0)):
            scale = s.t()[at].double()[..., None]
            off = (x.double() - y).abs() - before * (1.01 * y.abs() + (40 * U * y.abs().amax(2, keepdim=True) if before else 0.0)) - (40 * U * 2 * y.abs().amax(2, keepdim=True) if before else 0.0)
            if code == E4M3:
                bound = (x.double().abs().maximum(y.abs()) * 2.0 ** -4 * (1 + 2 * before) + scale * 2.0 ** -10)
            else:
                bound = scale * 0.5 * (1 + 2 * before) + 1e-7 * y.abs()
            assert bool((off <= bound * (1 + 1e-6)).all())


def test_a_serving_step_in_a_graph(example):
    """Rotation, write and attention captured once and replayed, with eager steps of another cache between the replays."""
    from paper_2508_03854_amd import TBE, rotary_frequencies
    tbe, N, H, K, dim, room = TBE([16], [8]), 6, 8, 2, 64, 700
    g = torch.Generator(device="cuda")
    g.manual_seed(10)
    freq, one = rotary_frequencies(dim), torch.arange(N + 1, device="cuda")
    starts = one * room
    ws = tbe.alloc_cache_attention_workspace(N, N, N * room, H, K, dim)
    caches = [tbe.alloc_cache(N * room, K, dim) for _ in range(2)]
    lengths = [torch.tensor([600, 3, 0, 90, 411, 250], device="cuda") for _ in range(2)]
    x = torch.randn(N, H + 2 * K, dim, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.zeros(N, H, dim, dtype=torch.bfloat16, device="cuda")

    def step(cache, lengths, out=None):
        q, k, v = x.split((H, K, K), 1)
        q, k = tbe.rotate_heads(q, k, lengths, freq, norm=True)
        tbe.cache_write(cache, k, v, starts[:-1] + lengths)
        lengths += 1
        return tbe.cache_attention(q, cache, one, starts, ws, k_lengths=lengths, out=out, stats=False)[0]

    step(caches[0], lengths[0], out)
    lengths[0] -= 1
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], lengths[0], out)
    for n in range(5):
        graph.replay()
        torch.cuda.synchronize()
        want = step(caches[1], lengths[1])
        assert torch.equal(out, want), n
        assert torch.equal(lengths[0], lengths[1])
        x.copy_(torch.randn(x.shape, generator=g, device="cuda").to(torch.bfloat16))
