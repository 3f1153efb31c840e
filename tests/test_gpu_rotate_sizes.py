"""Heads whose squares leave fp32's range or fall below it, with eps 0 and the smallest ones, normed and rotated, and the gradients, against the
definition in 64 bits.

Tolerances are those of tests/test_gpu_rotate.py: the power of two that a head is multiplied by rounds nothing but what lies 2^-126 below the head's
largest magnitude.  Half a unit of the subnormal numbers of the result's type (and of fp32, before) is added."""
import math

import pytest
import torch

from test_gpu_rotate import HALF, U, both, frequencies, turn

pytestmark = pytest.mark.gpu
SUB = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133 + 2.0 ** -149, torch.float16: 2.0 ** -24 + 2.0 ** -149}


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def close(got, ref, tol, dtype, what):
    err = (got.double() - ref).abs()
    tol = tol + HALF[dtype] * (ref.abs() + tol) + SUB[dtype]
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} over the bound, {got[bad][0].item():.6g} for {ref[bad][0].item():.6g} +- {tol[bad][0].item():.3g}"


def compare(tbe, x, dy, w, turned, eps, interleaved, what):
    """x, dy: [rows, heads, dim], the same for q and k (k: its heads the other way round)."""
    rows, heads, dim = x.shape
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + dim)
    p = torch.randint(-1000, 1000, (rows,), generator=g, device="cuda")
    f = frequencies(turned)
    eps = float(torch.tensor(eps))   # (as fp32 has it)
    how = dict(interleaved=interleaved, norm=True, eps=eps, q_weight=w, k_weight=w)
    xs, dys = (x, x.flip(1).contiguous()), (dy, dy.flip(1).contiguous())
    out = tbe.rotate_heads(*xs, p, f, **how)
    ws = tbe.alloc_rotate_workspace(rows, heads, heads, dim)
    grads = tbe.rotate_heads_backward(*dys, p, f, ws, q=xs[0], k=xs[1], **how)
    w64 = w.double()
    for i in range(2):
        x64, dy64 = xs[i].double(), dys[i].double()
        r = 1.0 / (x64.square().mean(2, keepdim=True) + eps).sqrt()
        h = x64 * r
        m, far = both((h * w64).abs(), p, f, interleaved, 1.0)
        close(out[i], turn(h * w64, p, f, interleaved, 1.0), 40 * U * m + 3 * 2.0 ** -53 * far, x.dtype, what + " y")
        G = turn(dy64, p, f, interleaved, 1.0, True)
        m, far = both(dy64.abs(), p, f, interleaved, 1.0)
        gerr = 3 * 2.0 ** -53 * far
        u = G * w64
        M, ferr = ((t * abs(w64) * h.abs()).mean(2, keepdim=True) for t in (m, gerr))
        close(grads[i], r * (u - h * (u * h).mean(2, keepdim=True)), r * (100 * U * (m * abs(w64) + h.abs() * M) + gerr * abs(w64) + h.abs() * ferr), x.dtype, what + " dx")
        close(grads[i + 2], (G * h).sum((0, 1)), ((156 + rows * heads / 2048) * U * m * h.abs() + gerr * h.abs()).sum((0, 1)), w.dtype, what + " dw")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_of_every_size(tbe, dtype, interleaved):
    """Neighbouring heads and rows up to 10^73 apart; eps 0 and so small that it matters only to the smallest heads, or only to those near it.  From
    2^-100 on heads up to 10^17."""
    for dim, turned in ((64, 64), (40, 24), (256, 256), (7, 4), (128, 128), (1, 0), (2, 2)):
        for eps in (0.0, 1e-45, 1e-38, 7.8e-31, 8e-31, 1e-20, 1e-6):
            g = torch.Generator(device="cuda")
            g.manual_seed(dim)
            size = torch.pow(10.0, torch.rand(50, 5, 1, generator=g, device="cuda", dtype=torch.float64) * (73 if eps < 2.0 ** -100 else 53) - 36.5)
            x = (torch.randn(50, 5, dim, generator=g, device="cuda").double() * size).to(dtype)
            dy = torch.randn(50, 5, dim, generator=g, device="cuda").to(dtype)
            w = torch.rand(dim, generator=g, device="cuda") + 0.5
            compare(tbe, x, dy, w, turned, eps, interleaved, f"{dim} {eps}")


@pytest.mark.parametrize("size", [1e-44, 1e-39, 1e-30, 1e-23, 2.6e-23, 1e-19, 1e19, 1.8e19, 3e38])
def test_on_either_side_of_the_range_of_squares(tbe, size):
    """All elements the same magnitude; results are +-1 turned.  (Upstream gradients are as large as the heads, so that the heads' own are finite.)"""
    for dtype in (torch.float32, torch.bfloat16)[:2 if size > 1e-40 else 1]:
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        sign = torch.randint(0, 2, (9, 3, 96), generator=g, device="cuda") * 2.0 - 1.0
        x = (sign.double() * size).to(dtype)
        assert bool((x != 0).all() and x.isfinite().all())
        dy = torch.randn(9, 3, 96, generator=g, device="cuda").to(dtype) * (1e-8 if size < 1e-30 else 1.0)
        compare(tbe, x, dy.to(dtype), torch.rand(96, generator=g, device="cuda") + 0.5, 96, 0.0, False, f"{size}")


def test_elements_of_very_different_sizes(tbe):
    """One large element, below or beyond the range of squares, and others 10^60 smaller: their squares count for nothing, and they come out as zeros."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    for large, small in ((1e30, 1e-30), (1e-24, 1e-44), (1e25, 1.0), (3e38, 3e37)):
        x = torch.randn(20, 2, 64, generator=g, device="cuda").clamp(-1, 1) * small
        x[:, :, 11] = large
        compare(tbe, x, torch.randn(20, 2, 64, generator=g, device="cuda"), torch.rand(64, generator=g, device="cuda") + 0.5, 48, 0.0, True, f"{large} {small}")


def test_ordinary_heads_beside_them_keep_their_bits(tbe):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    for dim, eps in ((32, 0.0), (40, 1e-6), (128, 0.0), (24, 1e-6), (40, 0.0), (7, 0.0)):
        x, dy = torch.randn(64, 8, dim, generator=g, device="cuda"), torch.randn(64, 8, dim, generator=g, device="cuda")
        p, f = torch.arange(64, device="cuda"), frequencies(dim // 2 * 2)
        ws = tbe.alloc_rotate_workspace(64, 8, 0, dim)
        want = tbe.rotate_heads(x, None, p, f, norm=True, eps=eps)[0]
        gwant = tbe.rotate_heads_backward(dy, None, p, f, ws, q=x, norm=True, eps=eps, params=False)[0]
        y = x.clone()
        y[::3, ::2] *= 1e-30
        y[1::5, 1::2] *= 1e30
        same = y == x
        got = tbe.rotate_heads(y, None, p, f, norm=True, eps=eps)[0]
        ggot = tbe.rotate_heads_backward(dy, None, p, f, ws, q=y, norm=True, eps=eps, params=False)[0]
        assert torch.equal(got[same], want[same]) and torch.equal(ggot[same], gwant[same])


def test_what_is_not_finite_and_zeros(tbe):
    """An infinite element: the others of its head become 0, itself not a number; zeros with eps 0 have no direction."""
    x = torch.randn(4, 3, 32, device="cuda")
    p = torch.arange(4, device="cuda")
    x[1, 2, 5] = math.inf
    x[2, 0, 7] = -math.inf
    x[3, 1] = 0.0
    y = tbe.rotate_heads(x, None, p, None, norm=True, eps=0.0)[0]
    for r, h, e in ((1, 2, 5), (2, 0, 7)):
        rest = y[r, h].clone()
        rest[e] = 0
        assert bool(y[r, h, e].isnan()) and bool((rest == 0).all())
    assert bool(y[3, 1].isnan().all())
    assert bool((tbe.rotate_heads(x, None, p, None, norm=True, eps=1e-45)[0][3, 1] == 0).all())
    big = torch.full((1, 1, 32), 1e25, device="cuda")
    assert bool((tbe.rotate_heads(big, None, p[:1], None, norm=True)[0] == 0).all())
