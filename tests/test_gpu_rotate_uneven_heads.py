"""Weights' gradients of the rotation where one matrix has few of the workgroups and many rows: q has 64 heads, k one.

The workgroups are shared out by heads, 3584 at most: k has 3584 / 65, rounded down 55 of them, 220 wavefronts, and of fp32 heads of 256 each takes two
rows at a time, one for either half of its lanes.  A lane then adds n / 440 terms one after the other, the halves 1, the four wavefronts 3, the 55
workgroups 2 and 32: fewer than n / 440 + 40 roundings, and 28 u of each term (tests/test_gpu_rotate.py).  Of q a wavefront takes two heads of a row at a time,
32 turns, of the 3528 workgroups left: n 32 / 14112 terms, and 3528 / 32 = 111 and 32 for those."""
import pytest
import torch

from test_gpu_rotate import U, both, frequencies, turn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("flipped", [False, True])
def test_one_head_beside_sixty_four(flipped):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    tbe = TBE([16], [8])
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n, dim = 100_003, 256
    p, f = torch.randint(0, 5000, (n,), generator=g, device="cuda"), frequencies(dim)
    one, dy = torch.randn(n, 1, dim, generator=g, device="cuda"), torch.randn(n, 1, dim, generator=g, device="cuda") + 1.0
    many, dmany = (torch.randn(1, 64, dim, generator=g, device="cuda").expand(n, 64, dim) for _ in range(2))   # (the same in every row: read, not written)
    w = torch.rand(dim, generator=g, device="cuda") + 0.5
    out = torch.empty(n, 64, dim, device="cuda")
    ws = tbe.alloc_rotate_workspace(n, 64, 1, dim)
    if flipped:
        grads = tbe.rotate_heads_backward(dy, dmany, p, f, ws, q=one, k=many, norm=True, q_weight=w, k_weight=w, grad_k=out)
        dw, dw_many = grads[2], grads[3]
    else:
        grads = tbe.rotate_heads_backward(dmany, dy, p, f, ws, q=many, k=one, norm=True, q_weight=w, k_weight=w, grad_q=out)
        dw, dw_many = grads[3], grads[2]

    def check(x, dy, p, got, terms, what):
        x, dy = x.double(), dy.double()
        h = x / (x.square().mean(2, keepdim=True) + 1e-6).sqrt()
        m, far = both(dy.abs(), p, f, False, 1.0)
        ref = (turn(dy, p, f, False, 1.0, True) * h).sum((0, 1))
        tol = (((28 + terms) * U * m + 3 * 2.0 ** -53 * far) * h.abs()).sum((0, 1))
        err = (got.double() - ref).abs()
        assert bool((err <= tol).all()), f"{what}: {(err / tol).max().item():.3g} of the bound"

    check(one, dy, p, dw, n / 440 + 40, "one")
    # every row of the 64 heads is the same: the turns back of all rows, added in 64 bits, are a turn by their mean
    c, s = (torch.zeros(dim // 2, dtype=torch.float64, device="cuda") for _ in range(2))
    for q in p.split(10_000):
        t = q.double()[:, None] * f
        c, s = c + t.cos().sum(0), s + t.sin().sum(0)
    x, y = many[0].double(), dmany[0].double()
    h = x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt()
    a, b = y[:, :dim // 2], y[:, dim // 2:]
    back = torch.cat((a * c + b * s, b * c - a * s), 1)
    m = (a.abs() + b.abs()) * n
    tol = ((28 + n * 32 / 14112 + 160) * U * torch.cat((m, m), 1) * h.abs()).sum(0) + 3 * 2.0 ** -53 * 5000 * n * (h.abs() * torch.cat((a.abs() + b.abs(), a.abs() + b.abs()), 1)).sum(0)
    err = (dw_many.double() - (back * h).sum(0)).abs()
    assert bool((err <= tol).all()), f"64 heads: {(err / tol).max().item():.3g} of the bound"
    torch.cuda.empty_cache()
