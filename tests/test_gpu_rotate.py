"""Heads normed and rotated by position, and the gradients, against the definition in 64 bits: both layouts, heads of every size and address, parts of a
head, apart rows, positions far off and below zero; gradients also against differences; values that are not finite; streams, graphs, refusals.

Tolerances, in units u = 2^-24 of the operands' magnitude.  A sum over a head: at most 16 terms one after the other and 6 steps of a tree, relative
to its own (positive) terms, so 1 / sqrt of it 12 and a few more, 20 with the two products that follow.  Sine and cosine: the angle, at most pi / 4, is
rounded once (0.4), the series' last steps (1.5), the amplitude and its product (1.5); the two products and their sum 2 more: 8 in all, and
the angle in 64 bits, three roundings: 3 2^-53 of its size.  Together fewer than 40 u (|z_a| + |z_b|).  Gradients: the turned gradient G 8 u, the norm 20 u, the mean
of u h 22 + 8 + 20 u of the mean of its magnitudes M, products: fewer than 100 u r (|u| + |h| M).  A weight's gradient over n terms: 28 u of a term, and of the
sum: at most n / 4096 + 16 terms one after the other in a lane (a wavefront takes every 4096th unit, and at most 8 heads more of a unit for itself), 3 + 2 for the
groups and wavefronts, 32 + 32 for the workgroups: 128 + n / 2048 u.  16-bit results: half a unit in their last place more."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}
# rows, q heads, k heads, head_dim, rotary_dim
SHAPES = [(1, 1, 1, 2, 2), (1, 1, 0, 1, 0), (3, 2, 1, 3, 2), (5, 0, 2, 7, 4), (33, 4, 4, 32, 32), (65, 8, 2, 128, 128), (17, 16, 4, 64, 24), (9, 3, 3, 80, 32),
          (129, 5, 1, 40, 40), (7, 1, 1, 256, 256), (4, 40, 8, 128, 64), (2, 33, 7, 100, 50), (31, 6, 2, 96, 94), (11, 2, 2, 250, 246), (1000, 3, 1, 72, 72),
          (257, 12, 12, 64, 2), (6, 8, 8, 192, 130), (2, 1024, 1, 16, 16), (70, 9, 3, 33, 18)]


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def matrix(g, rows, heads, dim, dtype, pad):
    """Rows and heads apart from each other (pad), from an address that is a multiple of one element only."""
    if heads == 0:
        return None
    row = heads * (dim + pad) + pad
    flat = torch.randn(rows * row + 1, generator=g, device="cuda").to(dtype)
    return flat[1 if pad else 0:].as_strided((rows, heads, dim), (row, dim + pad, 1))


def frequencies(turned, base=1e4):
    return torch.tensor([base ** (-2 * j / turned) for j in range(turned // 2)], dtype=torch.float64, device="cuda")


def pairs(turned, interleaved):
    j = torch.arange(turned // 2, device="cuda")
    return (2 * j, 2 * j + 1) if interleaved else (j, j + turned // 2)


def angles(positions, freq):
    return (positions.double()[:, None] * freq)[:, None]


def turn(x, positions, freq, interleaved, amplitude, back=False):
    a, b = pairs(2 * freq.numel(), interleaved)
    t = angles(positions, freq) * (-1 if back else 1)
    y = x.clone()
    y[..., a] = amplitude * (x[..., a] * t.cos() - x[..., b] * t.sin())
    y[..., b] = amplitude * (x[..., b] * t.cos() + x[..., a] * t.sin())
    return y


def both(mag, positions, freq, interleaved, amplitude):
    """|z_a| + |z_b| times the amplitude, and that times the angle."""
    a, b = pairs(2 * freq.numel(), interleaved)
    m, far = mag.clone(), torch.zeros_like(mag)
    m[..., a] = m[..., b] = abs(amplitude) * (mag[..., a] + mag[..., b])
    far[..., a] = far[..., b] = m[..., a] * angles(positions, freq).abs()
    return m, far


def close(got, ref, tol, dtype, what):
    err = (got.double() - ref).abs()
    tol = tol + HALF[dtype] * (ref.abs() + tol) + TINY[dtype]
    assert bool((err <= tol).all()), f"{what}: {(err - tol).max().item():.3g} over the bound, error {err.max().item():.3g}"


def check(tbe, rows, heads, dim, turned, dtype, params, pad, interleaved, norm, amplitude, span, index=torch.int64, seed=0, eps=1e-6):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + rows * 31 + dim)
    what = f"{rows} {heads} {dim} {turned}"
    positions = torch.randint(-span, span, (rows,), generator=g, device="cuda").to(index)
    freq = frequencies(turned) if turned else None
    f64 = freq if turned else torch.zeros(0, dtype=torch.float64, device="cuda")
    x = [matrix(g, rows, n, dim, dtype, pad) for n in heads]
    w = [torch.randn(dim, generator=g, device="cuda").mul_(0.3).add_(1).to(params) if norm and n else None for n in heads]
    dy = [matrix(g, rows, n, dim, dtype, pad) for n in heads]
    how = dict(interleaved=interleaved, amplitude=amplitude, norm=norm, eps=eps, q_weight=w[0], k_weight=w[1])
    out = tbe.rotate_heads(x[0], x[1], positions, freq, **how)
    ws = None
    if norm:
        ws = tbe.alloc_rotate_workspace(rows, heads[0], heads[1], dim)
        ws.fill_(255)
    grads = tbe.rotate_heads_backward(dy[0], dy[1], positions, freq, ws, q=x[0] if norm else None, k=x[1] if norm else None, **how)
    again = tbe.rotate_heads_backward(dy[0], dy[1], positions, freq, ws, q=x[0] if norm else None, k=x[1] if norm else None, **how)
    amplitude = float(torch.tensor(amplitude))
    for i, n in enumerate(heads):
        if n == 0:
            assert out[i] is None and grads[i] is None and grads[i + 2] is None
            continue
        x64, dy64, w64 = x[i].double(), dy[i].double(), 1.0 if w[i] is None else w[i].double()
        r = 1.0 / (x64.square().mean(2, keepdim=True) + eps).sqrt()
        z = x64 * r * w64 if norm else x64
        m, far = both(z.abs(), positions, f64, interleaved, amplitude)
        close(out[i], turn(z, positions, f64, interleaved, amplitude), 40 * U * m + 3 * 2.0 ** -53 * far, dtype, what + " y")
        G = turn(dy64, positions, f64, interleaved, amplitude, True)
        m, far = both(dy64.abs(), positions, f64, interleaved, amplitude)
        gerr = 3 * 2.0 ** -53 * far
        assert torch.equal(grads[i], again[i])
        if not norm:
            close(grads[i], G, 8 * U * m + gerr, dtype, what + " dx")
            continue
        h, u = x64 * r, G * w64
        M = (m * abs(w64) * h.abs()).mean(2, keepdim=True)
        ferr = (gerr * abs(w64) * h.abs()).mean(2, keepdim=True)
        close(grads[i], r * (u - h * (u * h).mean(2, keepdim=True)), r * (100 * U * (m * abs(w64) + h.abs() * M) + gerr * abs(w64) + h.abs() * ferr), dtype, what + " dx")
        close(grads[i + 2], (G * h).sum((0, 1)), ((156 + rows * n / 2048) * U * m * h.abs() + gerr * h.abs()).sum((0, 1)), params, what + " dw")
        assert torch.equal(grads[i + 2], again[i + 2])


@pytest.mark.parametrize("dtype,params", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
def test_against_64_bits(tbe, dtype, params, interleaved, norm, pad):
    for rows, H, K, dim, turned in SHAPES:
        check(tbe, rows, (H, K), dim, turned, dtype, params, pad, interleaved, norm, 1.0, 1000)


@pytest.mark.parametrize("span,index", [(2 ** 31 - 1, torch.int32), (2 ** 33, torch.int64), (1, torch.int64)])
def test_far_positions_and_amplitudes(tbe, span, index):
    for amplitude in (1.25, -0.5, 0.0):
        check(tbe, 77, (4, 2), 64, 64, torch.float32, torch.float32, 0, False, True, amplitude, span, index)
        check(tbe, 77, (4, 2), 64, 48, torch.float32, torch.float32, 0, True, False, amplitude, span, index)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_rows(tbe, dtype):
    """More units than wavefronts, and rows' heads in pieces."""
    check(tbe, 30_011, (6, 2), 64, 64, dtype, torch.float32, 0, False, True, 1.0, 30_000)
    check(tbe, 3, (1000, 24), 128, 128, dtype, torch.float32, 0, True, True, 1.0, 30_000)


def test_a_turn_keeps_lengths_and_differences(tbe):
    """q . k depends on the difference of the positions only: 64 products of magnitude up to |q||k| / 8 each, 40 u of each factor."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, k = (torch.randn(1, 1, 64, generator=g, device="cuda").expand(200, 1, 64).contiguous() for _ in range(2))
    p = torch.arange(200, device="cuda") * 1_000_003
    f = frequencies(64)
    yq, yk = tbe.rotate_heads(q, k, p, f)
    _, back = tbe.rotate_heads(None, k, p - 17, f)
    dots = (yq.double() * back.double()).sum(2)
    assert (dots - dots[0]).abs().max() <= 4 * 40 * U * (q[0].double().abs().sum() * k[0].double().abs().max() * 2)
    assert (yq.double().norm(dim=2) - q.double().norm(dim=2)).abs().max() <= 40 * U * 2 * q[0].double().abs().sum()


def test_gradients_against_differences(tbe):
    """Central differences of the formula in 64 bits, step 1e-4: off by the third derivative times 1e-8 / 6 and by 2^-53 1e4 of the sum's size."""
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    rows, H, dim, turned = 3, 2, 10, 6
    x, w, dy = torch.randn(rows, H, dim, generator=g, device="cuda"), torch.rand(dim, generator=g, device="cuda") + 0.5, torch.randn(rows, H, dim, generator=g, device="cuda")
    p, f = torch.tensor([3, 0, -7], device="cuda"), frequencies(turned)

    def loss(x, w):
        return (turn(x / (x.square().mean(2, keepdim=True) + 1e-6).sqrt() * w, p, f, False, 1.5) * dy.double()).sum()

    gx, _, gw, _ = tbe.rotate_heads_backward(dy, None, p, f, tbe.alloc_rotate_workspace(rows, H, 0, dim), q=x, norm=True, q_weight=w, amplitude=1.5)
    for got, leaf, other in ((gx, x, w), (gw, w, x)):
        for i in range(leaf.numel()):
            e = torch.zeros(leaf.numel(), dtype=torch.float64, device="cuda")
            e[i] = 1e-4
            e = e.view(leaf.shape)
            a, b = ((loss(leaf.double() + s * e, other.double()) if leaf is x else loss(other.double(), leaf.double() + s * e)) for s in (1, -1))
            assert abs(float((a - b) / 2e-4) - float(got.view(-1)[i])) < 1e-5


def test_in_place_and_what_lies_between(tbe):
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    p, f = torch.arange(50, device="cuda"), frequencies(20)
    for dtype in (torch.float32, torch.bfloat16):
        all_ = torch.randn(50, 9, 24, generator=g, device="cuda").to(dtype)
        q, k, v = all_.split((4, 2, 3), 1)
        before = v.clone()
        for norm in (False, True):
            want = tbe.rotate_heads(q, k, p, f, norm=norm)
            buf = torch.full((50, 9, 26), 7.0, dtype=dtype, device="cuda")
            got = tbe.rotate_heads(q, k, p, f, norm=norm, q_out=buf[:, 1:5, 1:25], k_out=buf[:, 6:8, 1:25])
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            mask = torch.ones(50, 9, 26, dtype=torch.bool, device="cuda")
            mask[:, 1:5, 1:25] = mask[:, 6:8, 1:25] = False
            assert bool((buf[mask] == 7).all())
            ws = tbe.alloc_rotate_workspace(50, 4, 2, 24)
            gwant = tbe.rotate_heads_backward(q, k, p, f, ws, q=k.repeat(1, 2, 1) if norm else None, k=q[:, :2].contiguous() if norm else None, norm=norm)
            over = all_.clone()
            oq, ok, _ = over.split((4, 2, 3), 1)
            ggot = tbe.rotate_heads_backward(oq, ok, p, f, ws, q=k.repeat(1, 2, 1) if norm else None, k=q[:, :2].contiguous() if norm else None, norm=norm, grad_q=oq, grad_k=ok)
            assert all(torch.equal(a, b) for a, b in zip(ggot[:2], gwant[:2])) and torch.equal(over[:, 6:], before)
        want = tbe.rotate_heads(q, k, p, f, norm=True)
        tbe.rotate_heads(q, k, p, f, norm=True, q_out=q, k_out=k)
        assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, before)


def test_matrices_by_head(tbe):
    """[heads][rows][dim] in memory."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    q = torch.randn(5, 40, 32, generator=g, device="cuda").to(torch.bfloat16)
    p, f = torch.arange(40, device="cuda", dtype=torch.int32), frequencies(32)
    out = torch.empty_like(q)
    tbe.rotate_heads(q.transpose(0, 1), None, p, f, q_out=out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1), tbe.rotate_heads(q.transpose(0, 1).contiguous(), None, p, f)[0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_values_that_are_not_finite_stay_where_they_are(tbe, interleaved):
    """Without norm only a pair's two elements; elements that are not turned pass through.  With norm a head, and no other."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    for dim, turned in ((64, 64), (64, 24), (40, 38), (24, 0)):
        x = torch.randn(6, 3, dim, generator=g, device="cuda")
        p, f = torch.arange(6, device="cuda") + 1, frequencies(turned) if turned else None
        clean = tbe.rotate_heads(x, None, p, f, interleaved=interleaved)[0]
        normed = tbe.rotate_heads(x, None, p, f, interleaved=interleaved, norm=True)[0]
        for e in range(dim):
            for bad in (math.inf, math.nan):
                y = x.clone()
                y[2, 1, e] = bad
                got = tbe.rotate_heads(y, None, p, f, interleaved=interleaved)[0]
                hit = torch.zeros_like(x, dtype=torch.bool)
                hit[2, 1, e] = True
                if e < turned:
                    hit[2, 1, e ^ 1 if interleaved else (e + turned // 2) % turned] = True
                assert torch.equal(got[~hit], clean[~hit]) and not bool(torch.isfinite(got[2, 1, e]))
                if e >= turned:
                    assert torch.equal(got[2, 1, e].isnan(), y[2, 1, e].isnan())
        y = x.clone()
        y[4, 2, dim - 1] = math.nan
        got = tbe.rotate_heads(y, None, p, f, interleaved=interleaved, norm=True)[0]
        assert bool(got[4, 2].isnan().all())
        got[4, 2] = normed[4, 2]
        assert torch.equal(got, normed)


def test_zero_heads_and_no_rows(tbe):
    p, f = torch.arange(3, device="cuda"), frequencies(8)
    x = torch.zeros(3, 2, 8, device="cuda")
    assert bool((tbe.rotate_heads(x, None, p, f, norm=True)[0] == 0).all())
    gx, _, gw, _ = tbe.rotate_heads_backward(torch.ones(3, 2, 8, device="cuda"), None, p, f, tbe.alloc_rotate_workspace(3, 2, 0, 8), q=x, norm=True)
    assert bool(torch.isfinite(gx).all()) and bool((gw == 0).all())
    none = x[:0]
    out = tbe.rotate_heads(none, none, p[:0], f, norm=True)
    assert out[0].shape == (0, 2, 8) and out[1].shape == (0, 2, 8)
    ws = tbe.alloc_rotate_workspace(0, 2, 2, 8)
    got = tbe.rotate_heads_backward(none, none, p[:0], f, ws, q=none, k=none, norm=True)
    assert bool((got[2] == 0).all()) and bool((got[3] == 0).all())
    tbe.rotate_heads_backward(none, none, p[:0], f)


def test_on_a_stream_and_in_a_graph(tbe):
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    q, k = torch.randn(100, 4, 64, generator=g, device="cuda"), torch.randn(100, 2, 64, generator=g, device="cuda")
    w = torch.rand(64, generator=g, device="cuda")
    p, f = torch.arange(100, device="cuda"), frequencies(64)
    ws = tbe.alloc_rotate_workspace(100, 4, 2, 64)
    outs = [torch.zeros_like(t) for t in (q, k, q, k)] + [torch.zeros_like(w), torch.zeros_like(w)]

    def work(stream=None):
        tbe.rotate_heads(q, k, p, f, norm=True, q_weight=w, k_weight=w, q_out=outs[0], k_out=outs[1], stream=stream)
        tbe.rotate_heads_backward(outs[0], outs[1], p, f, ws, q=q, k=k, norm=True, q_weight=w, k_weight=w, grad_q=outs[2], grad_k=outs[3], grad_q_weight=outs[4],
                                  grad_k_weight=outs[5], stream=stream)

    work()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    s = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    work(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for n in range(3):
        q.mul_(1.5)
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, got)), n


def test_refusals(tbe):
    from paper_2508_03854_amd import TbeError, binding as B
    q, k = torch.randn(4, 2, 16, device="cuda"), torch.randn(4, 1, 16, device="cuda")
    p, f, w = torch.arange(4, device="cuda"), frequencies(16), torch.ones(16, device="cuda")
    ok = lambda **kw: tbe.rotate_heads(q, k, p, f, **kw)  # noqa: E731
    ok()
    for bad, kind in ((lambda: tbe.rotate_heads(None, None, p, f), ValueError), (lambda: tbe.rotate_heads(q[:, 0], k, p, f), ValueError),
                      (lambda: tbe.rotate_heads(q, k[:3], p, f), ValueError), (lambda: tbe.rotate_heads(q, k.half(), p, f), ValueError),
                      (lambda: tbe.rotate_heads(q, k[..., :8], p, f), ValueError), (lambda: tbe.rotate_heads(q, k, p[:3], f), ValueError),
                      (lambda: tbe.rotate_heads(q, k, p.float(), f), TypeError), (lambda: tbe.rotate_heads(q, k, p, f.float()), TypeError),
                      (lambda: tbe.rotate_heads(q.double(), None, p, f), TypeError), (lambda: tbe.rotate_heads(q.cpu(), None, p, f), ValueError),
                      (lambda: tbe.rotate_heads(q.transpose(1, 2), None, p, f), ValueError), (lambda: ok(q_weight=w), ValueError),
                      (lambda: ok(norm=True, q_weight=w[:8]), ValueError), (lambda: ok(norm=True, q_weight=w, k_weight=w.half()), TypeError),
                      (lambda: ok(q_out=q[:3]), ValueError), (lambda: tbe.rotate_heads(None, k, p, f, q_out=q), ValueError),
                      (lambda: tbe.rotate_heads_backward(q, k, p, f, norm=True), ValueError), (lambda: tbe.rotate_heads_backward(q, k, p, f, grad_q_weight=w), ValueError)):
        with pytest.raises(kind):
            bad()
    big = torch.zeros(1, 1, 258, device="cuda")
    for bad, status in ((lambda: tbe.rotate_heads(big, None, p[:1], None), B.ESHAPE), (lambda: tbe.rotate_heads(q[..., :8], None, p, f), B.ESHAPE),
                        (lambda: tbe.rotate_heads(torch.zeros(1, 1025, 2, device="cuda"), None, p[:1], None), B.ESHAPE),
                        (lambda: ok(amplitude=math.inf), B.EINVAL), (lambda: ok(norm=True, eps=-1.0), B.EINVAL), (lambda: ok(norm=True, eps=math.nan), B.EINVAL),
                        (lambda: tbe.rotate_heads(q, None, p, f, q_out=q.new_zeros(16).expand(4, 2, 16)), B.EINVAL),
                        (lambda: tbe.rotate_heads(q.new_zeros(16).expand(4, 2, 16), None, p, f, q_out=None) and tbe.rotate_heads_backward(q, None, p, f, None, q=q, norm=True), B.EINVAL),
                        (lambda: tbe.rotate_heads_backward(q, None, p, f, torch.empty(256, dtype=torch.uint8, device="cuda"), q=q, norm=True), B.EWORKSPACE)):
        with pytest.raises(TbeError) as e:
            bad()
        assert e.value.status == status
    same = q.clone()
    apart = torch.zeros(4, 2, 32, device="cuda")
    with pytest.raises(TbeError):   # one matrix, two strides
        tbe.rotate_heads(apart[..., :16], None, p, f, q_out=apart.view(-1)[:128].view(4, 2, 16))
    assert torch.equal(q, same)
