"""Layer norm and its gradients against the definition in 64 bits: every way a row is shared among lanes, odd widths at odd addresses,
apart rows, one row and none, constant rows, both parameter types; gradients also against differences; refusals.

Tolerances.  fp32 results: a sum of n terms in fp32, a few dozen of them one after the other and the rest as a tree, is off by at most
(32 + 2 log2 n) 2^-24 of the sum of its terms' magnitudes; a handful of further roundings follow.  80 units of 2^-24 of the operands'
magnitude bound that with room.  Mean and rstd carry it to (x - mean) rstd, whose magnitude is |h| + |mean| rstd.  16-bit results: half a unit
in the last place of the result more (at most 2^-8 bfloat16, 2^-11 binary16 of it, and for binary16 the spacing of its subnormals).  A column sum over
r rows: at most r / 4 of them one after the other, bounded by 2^-24 (80 + sqrt r) of the magnitudes' sum."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -24}
SHAPES = [(1, 1), (3, 2), (65, 7), (1, 33), (1000, 8), (517, 16), (64, 31), (129, 64), (33, 100), (7, 128), (2049, 132), (70, 255), (9, 256),
          (257, 260), (5, 511), (31, 513), (40, 1000), (6, 1021), (77, 1024), (3, 1025), (18, 2048), (2, 2049), (5, 4097), (3, 8191), (4, 8192),
          (40000, 24), (6000, 300)]


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def matrix(g, rows, cols, dtype, pad, mul=1.0, add=0.0):
    """Rows `pad` elements apart from each other, from an address that is a multiple of one element only."""
    n = rows * (cols + pad) + 1
    flat = torch.randn(n, generator=g, device="cuda").mul_(mul).add_(add).to(dtype)
    return flat[1 if pad else 0:][:rows * (cols + pad)].view(rows, cols + pad)[:, :cols]


def inputs(rows, cols, dtype, params, pad, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + rows * 10007 + cols)
    w = torch.randn(cols, generator=g, device="cuda").mul_(0.5).add_(1.0).to(params)
    b = torch.randn(cols, generator=g, device="cuda").to(params)
    return matrix(g, rows, cols, dtype, pad, 0.8, 0.3), matrix(g, rows, cols, dtype, pad), w, b


def close(got, ref, mag, units, dtype, what):
    err = (got.double() - ref).abs()
    tol = units * U * mag + HALF[dtype] * ref.abs() * 1.01 + TINY[dtype]
    assert bool((err <= tol).all()), f"{what}: {(err - tol).max().item():.3g} over the bound, error {err.max().item():.3g}"


@pytest.mark.parametrize("dtype,params", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
                                          (torch.float16, torch.float16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("pad", [0, 5])
def test_forward_and_gradients_against_64_bits(tbe, dtype, params, pad):
    for rows, cols in SHAPES:
        x, dy, w, b = inputs(rows, cols, dtype, params, pad)
        what = f"{rows}x{cols}"
        y, mean, rstd = tbe.layer_norm(x, w, b, eps=1e-3)
        x64, dy64, w64, b64 = x.double(), dy.double(), w.double(), b.double()
        m = x64.mean(1, keepdim=True)
        r = 1.0 / ((x64 - m).square().mean(1, keepdim=True) + 1e-3).sqrt()
        h = (x64 - m) * r
        big = x64.abs().amax(1, keepdim=True)
        close(mean, m[:, 0], big[:, 0], 80, torch.float32, what + " mean")
        close(rstd, r[:, 0], r[:, 0] * (1 + big[:, 0] * r[:, 0]), 80, torch.float32, what + " rstd")
        hmag = h.abs() * (2 + big * r) + big * r
        close(y, h * w64 + b64, hmag * w64.abs() + b64.abs(), 80, dtype, what + " y")
        # the gradients from the very statistics that the backward is given
        m, r = mean.double()[:, None], rstd.double()[:, None]
        h, gw = (x64 - m) * r, dy64 * w64
        dx = r * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
        hm = h.abs() + big * r
        mag = r * (gw.abs() + gw.abs().mean(1, keepdim=True) + hm * (gw.abs() * hm).mean(1, keepdim=True))
        ws = tbe.alloc_layer_norm_workspace(rows, cols)
        ws.fill_(255)
        gx, gwt, gbt = tbe.layer_norm_backward(dy, x, w, mean, rstd, ws)
        close(gx, dx, mag, 80, dtype, what + " dx")
        close(gwt, (dy64 * h).sum(0), (dy64.abs() * hm).sum(0), 80 + rows ** 0.5, params, what + " dw")
        close(gbt, dy64.sum(0), dy64.abs().sum(0), 80 + rows ** 0.5, params, what + " db")
        again = tbe.layer_norm_backward(dy, x, w, mean, rstd, ws)
        assert all(torch.equal(p, q) for p, q in zip((gx, gwt, gbt), again)), what


def test_without_parameters_and_in_place(tbe):
    x, dy, _, _ = inputs(100, 36, torch.float32, torch.float32, 0)
    one, zero = torch.ones(36, device="cuda"), torch.zeros(36, device="cuda")
    y, mean, rstd = tbe.layer_norm(x, one, zero)
    y2, none, _ = tbe.layer_norm(x, stats=False)
    assert none is None and torch.equal(y, y2)
    ws = tbe.alloc_layer_norm_workspace(100, 36)
    gx, gw, gb = tbe.layer_norm_backward(dy, x, one, mean, rstd, ws)
    gx2, nw, nb = tbe.layer_norm_backward(dy, x, None, mean, rstd, None, params=False)
    assert nw is None and nb is None and torch.equal(gx, gx2)
    _, gw2, nb = tbe.layer_norm_backward(dy, x, None, mean, rstd, ws, params=False, grad_weight=torch.empty(36, device="cuda"))
    assert nb is None and torch.equal(gw, gw2)
    over = dy.clone()
    tbe.layer_norm_backward(over, x, one, mean, rstd, None, grad_x=over, params=False)
    assert torch.equal(over, gx)
    over = x.clone()
    tbe.layer_norm(over, one, zero, out=over)
    assert torch.equal(over, y)


def test_rows_apart_leave_what_lies_between(tbe):
    for dtype in (torch.float32, torch.bfloat16):
        for cols in (5, 64, 99, 1030):
            x, dy, w, b = inputs(50, cols, dtype, torch.float32, 3)
            buf = torch.full((50, cols + 6), 7.0, dtype=dtype, device="cuda")
            ref, mean, rstd = tbe.layer_norm(x, w, b)
            tbe.layer_norm(x, w, b, out=buf[:, 1:cols + 1])
            assert torch.equal(buf[:, 1:cols + 1], ref) and bool((buf[:, 0] == 7).all()) and bool((buf[:, cols + 1:] == 7).all())
            ws = tbe.alloc_layer_norm_workspace(50, cols)
            gx = tbe.layer_norm_backward(dy, x, w, mean, rstd, ws)[0]
            tbe.layer_norm_backward(dy, x, w, mean, rstd, ws, grad_x=buf[:, 1:cols + 1])
            assert torch.equal(buf[:, 1:cols + 1], gx) and bool((buf[:, 0] == 7).all()) and bool((buf[:, cols + 1:] == 7).all())


def test_constant_rows_large_offsets_and_non_finite_rows(tbe):
    x = torch.full((8, 96), 3.25, device="cuda")
    y, mean, rstd = tbe.layer_norm(x, eps=1e-5)
    assert bool((y == 0).all()) and bool((mean == 3.25).all())
    # a spread of 1 around 1000: variance as a difference of squares would lose half its bits
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(64, 200, generator=g, device="cuda") + 1000.0
    ref = torch.nn.functional.layer_norm(x.double(), (200,))
    assert (tbe.layer_norm(x, stats=False)[0].double() - ref).abs().max() < 80 * U * 1000
    x[3, 17], x[5, 0], x[9, 199] = float("nan"), float("inf"), float("-inf")
    y = tbe.layer_norm(x, stats=False)[0]
    bad = ~torch.isfinite(y).all(1)
    assert bad.nonzero()[:, 0].tolist() == [3, 5, 9] and (y[~bad].double() - ref[~bad]).abs().max() < 80 * U * 1000


def test_gradients_against_differences(tbe):
    """The loss sum(y * dy) in 64 bits at x +- d e: a central difference is off by d^2 / 6 of the third derivative, here below 1e-6 of
    the gradient's scale; the kernels' fp32 result is held to 1e-5 of it."""
    x, dy, w, b = inputs(6, 12, torch.float32, torch.float32, 0)
    _, mean, rstd = tbe.layer_norm(x, w, b, eps=1e-3)
    got = tbe.layer_norm_backward(dy, x, w, mean, rstd, tbe.alloc_layer_norm_workspace(6, 12))

    def loss(x, w, b):
        m = x.mean(1, keepdim=True)
        return (((x - m) / ((x - m).square().mean(1, keepdim=True) + 1e-3).sqrt() * w + b) * dy.double()).sum()

    at = [x.double(), w.double(), b.double()]
    for k, grad in enumerate(got):
        num = torch.zeros_like(at[k]).view(-1)
        for e in range(num.numel()):
            side = []
            for d in (1e-4, -1e-4):
                p = [t.clone() for t in at]
                p[k].view(-1)[e] += d
                side.append(loss(*p))
            num[e] = (side[0] - side[1]) / 2e-4
        assert (num - grad.double().view(-1)).abs().max() <= 1e-5 * max(1.0, num.abs().max().item())


def test_no_rows(tbe):
    x = torch.empty(0, 40, device="cuda")
    y, mean, rstd = tbe.layer_norm(x)
    gx, gw, gb = tbe.layer_norm_backward(x, x, torch.ones(40, device="cuda"), mean, rstd, tbe.alloc_layer_norm_workspace(0, 40))
    assert y.shape == (0, 40) and bool((gw == 0).all()) and bool((gb == 0).all())


def test_on_another_stream_and_in_a_graph(tbe):
    x, dy, w, b = inputs(3000, 128, torch.bfloat16, torch.float32, 0)
    ws = tbe.alloc_layer_norm_workspace(3000, 128)
    ref = tbe.layer_norm(x, w, b)
    gref = tbe.layer_norm_backward(dy, x, w, ref[1], ref[2], ws)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [torch.empty_like(t) for t in (*ref, *gref)]

    def both(stream=None):
        tbe.layer_norm(x, w, b, out=got[0], mean=got[1], rstd=got[2], stream=stream)
        tbe.layer_norm_backward(dy, x, w, got[1], got[2], ws, grad_x=got[3], grad_weight=got[4], grad_bias=got[5], stream=stream)

    both(s)
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, (*ref, *gref)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (*ref, *gref)))


def test_timing_records(tbe):
    x, dy, w, b = inputs(10, 16, torch.float32, torch.float32, 0)
    tbe.timing_enable(True)
    _, m, r = tbe.layer_norm(x, w, b)
    tbe.layer_norm_backward(dy, x, w, m, r, tbe.alloc_layer_norm_workspace(10, 16))
    names = [n for n, _ in tbe.timing_read()]
    tbe.timing_enable(False)
    assert names == ["layer_norm", "layer_norm_backward", "layer_norm_params"]


def test_refusals(tbe):
    from paper_2508_03854_amd import binding
    x, dy, w, b = inputs(10, 16, torch.float32, torch.float32, 0)
    _, m, r = tbe.layer_norm(x, w, b)
    ws = tbe.alloc_layer_norm_workspace(10, 16)

    def status(f):
        with pytest.raises(binding.TbeError) as e:
            f()
        return e.value.status

    for eps in (-1.0, float("nan"), float("inf")):
        assert status(lambda: tbe.layer_norm(x, w, b, eps=eps)) == binding.EINVAL
    wide = torch.zeros(1, 8193, device="cuda")
    assert status(lambda: tbe.layer_norm(wide)) == binding.ESHAPE
    assert status(lambda: tbe.layer_norm(torch.zeros(2, 0, device="cuda"))) == binding.ESHAPE
    assert status(lambda: tbe.layer_norm(torch.zeros(1, 16, device="cuda").expand(10, 16))) == binding.EINVAL      # rows on top of each other
    assert status(lambda: tbe.layer_norm_backward(dy, x, w, m, r, None)) == binding.EINVAL
    assert status(lambda: tbe.layer_norm_backward(dy, x, w, m, r, ws[:0])) in (binding.EINVAL, binding.EWORKSPACE)
    assert status(lambda: tbe.layer_norm_backward(dy, x, w, m, r, ws[1:])) == binding.EINVAL
    assert status(lambda: tbe.layer_norm_workspace_bytes(-1, 16)) == binding.ESHAPE
    for bad in (lambda: tbe.layer_norm(x.cpu()), lambda: tbe.layer_norm(x.t()), lambda: tbe.layer_norm(x, w[:-1], b),
                lambda: tbe.layer_norm(x, w, b, out=torch.empty(10, 17, device="cuda")), lambda: tbe.layer_norm(x[0]),
                lambda: tbe.layer_norm_backward(dy[:9], x, w, m, r, ws)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: tbe.layer_norm(x.double()), lambda: tbe.layer_norm(x, w.half(), b), lambda: tbe.layer_norm(x, w, b, mean=m.half()),
                lambda: tbe.layer_norm_backward(dy, x, w, m, r, ws, grad_bias=b.half())):
        with pytest.raises(TypeError):
            bad()
    L = binding.load_library()
    assert L.tbe_layer_norm(tbe._h, x.data_ptr(), 16, 3, 10, 16, None, None, 0, 1e-5, x.data_ptr(), 16, None, None, None) == binding.EDTYPE
    assert L.tbe_layer_norm(None, x.data_ptr(), 16, 0, 10, 16, None, None, 0, 1e-5, x.data_ptr(), 16, None, None, None) == binding.EINVAL
    assert L.tbe_layer_norm(tbe._h, x.data_ptr(), 16, 0, 10, 16, None, None, 0, 1e-5, x.data_ptr() + 2, 16, None, None, None) == binding.EINVAL
