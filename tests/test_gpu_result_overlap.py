"""Results whose rows lie on their own heads, on each other or, shifted, on what they are made from are refused; layouts that only look alike, and results
that are their own sources, run."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


def refused(call):
    from paper_2508_03854_amd import TbeError, binding
    with pytest.raises(TbeError) as e:
        call()
    assert e.value.status == binding.EINVAL


# strides of [5 rows][4 heads][32]: rows that lie on the next row's heads
CROSSED = [(32, 32), (64, 32), (96, 32), (64, 96), (32, 64)]
# ... and that do not: rows of heads, heads of rows, rows between another row's heads
APART = [(128, 32), (32, 160), (176, 48), (48, 640), (200, 32), (256, 64)]


def test_rotation(tbe):
    x = torch.randn(5, 4, 32, device="cuda")
    p, f = torch.arange(5, device="cuda"), torch.ones(16, dtype=torch.float64, device="cuda")
    flat = torch.zeros(4096, device="cuda")
    for s in CROSSED:
        y = flat.as_strided((5, 4, 32), (*s, 1))
        refused(lambda: tbe.rotate_heads(x, None, p, f, q_out=y))
        refused(lambda: tbe.rotate_heads(None, x, p, f, k_out=y))
        refused(lambda: tbe.rotate_heads_backward(x, None, p, f, grad_q=y))
        refused(lambda: tbe.rotate_heads_backward(None, x, p, f, grad_k=y))
    assert not flat.any()
    want = tbe.rotate_heads(x, None, p, f)[0]
    for s in APART:
        y = flat.as_strided((5, 4, 32), (*s, 1))
        assert torch.equal(tbe.rotate_heads(x, None, p, f, q_out=y)[0], want)


def test_caches(tbe):
    from paper_2508_03854_amd import Cache
    x, slots = torch.randn(5, 4, 32, device="cuda"), torch.arange(5, device="cuda")
    cache = tbe.alloc_cache(5, 4, 32)
    tbe.cache_write(cache, x, x, slots)
    want = tbe.cache_read(cache, slots)[0]
    flat = torch.zeros(4096, device="cuda")
    codes = [torch.zeros(4096, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    good = tbe.alloc_cache(5, 4, 32)
    for s in CROSSED:
        y = flat.as_strided((5, 4, 32), (*s, 1))
        refused(lambda: tbe.cache_read(cache, slots, k_out=y, v_out=torch.empty_like(x)))
        refused(lambda: tbe.cache_read(cache, slots, k_out=torch.empty_like(x), v_out=y))
        c = codes[0].as_strided((5, 4, 32), (*s, 1))
        refused(lambda: tbe.cache_write(Cache(c, good.v, good.k_scales, good.v_scales), x, x, slots))
        refused(lambda: tbe.cache_write(Cache(good.k, c, good.k_scales, good.v_scales), x, x, slots))
    assert not flat.any() and not codes[0].view(torch.uint8).any() and not good.k.view(torch.uint8).any()
    for s in APART:
        y = flat.as_strided((5, 4, 32), (*s, 1))
        assert torch.equal(tbe.cache_read(cache, slots, k_out=y, v_out=torch.empty_like(x))[0], want)
        if s[0] % 16 == 0 and s[1] % 16 == 0:
            k, v = (c.as_strided((5, 4, 32), (*s, 1)) for c in codes)
            tbe.cache_write(Cache(k, v, good.k_scales, good.v_scales), x, x, slots)
            assert torch.equal(k.float(), cache.k.float()) and torch.equal(v.float(), cache.v.float())


def test_attention(tbe):
    x, off = torch.randn(5, 4, 32, device="cuda"), torch.tensor([0, 5], device="cuda")
    cache = tbe.alloc_cache(5, 4, 32)
    tbe.cache_write(cache, x, x, torch.arange(5, device="cuda"))
    flat = torch.zeros(4096, device="cuda")
    ws, cws = tbe.alloc_attention_workspace(1, 5, 5, 4, 4, 32), tbe.alloc_cache_attention_workspace(1, 5, 5, 4, 4, 32)
    for s in CROSSED:
        y = flat.as_strided((5, 4, 32), (*s, 1))
        refused(lambda: tbe.attention(x, x, x, off, off, ws, out=y))
        refused(lambda: tbe.cache_attention(x, cache, off, off, cws, out=y))
    assert not flat.any()
    want, cwant = tbe.attention(x, x, x, off, off, ws)[0], tbe.cache_attention(x, cache, off, off, cws)[0]
    for s in APART:
        if s[0] % 4 == 0 and s[1] % 4 == 0:
            y = flat.as_strided((5, 4, 32), (*s, 1))
            assert torch.equal(tbe.attention(x, x, x, off, off, ws, out=y)[0], want)
            assert torch.equal(tbe.cache_attention(x, cache, off, off, cws, out=y)[0], cwant)


def test_rotations_of_one_memory(tbe):
    p, f = torch.arange(6, device="cuda"), torch.ones(16, dtype=torch.float64, device="cuda")
    ws = tbe.alloc_rotate_workspace(6, 4, 2, 32)
    wide = torch.randn(8, 12, 32, device="cuda")
    before = wide.clone()
    q, k = wide[:6, :4], wide[:6, 4:6]
    refused(lambda: tbe.rotate_heads(q, k, p, f, q_out=wide[1:7, :4]))        # q's rows, one further on
    refused(lambda: tbe.rotate_heads(q, k, p, f, q_out=wide[:6, 1:5]))        # its heads
    refused(lambda: tbe.rotate_heads(q, k, p, f, k_out=wide[:6, 3:5]))        # a head of q
    refused(lambda: tbe.rotate_heads(q, k, p, f, q_out=wide[2:8, 4:8]))       # k's later rows
    refused(lambda: tbe.rotate_heads(q, k, p, f, q_out=wide[:6, 6:10], k_out=wide[:6, 9:11]))
    refused(lambda: tbe.rotate_heads(q, q, p, f, q_out=q, k_out=q))
    refused(lambda: tbe.rotate_heads(k, k, p, f, q_out=k))                    # made into q's result while it is read for k's
    one = wide.view(-1)[5:5 + 6 * 32].view(6, 1, 32)
    refused(lambda: tbe.rotate_heads(one, None, p, f, q_out=wide.view(-1)[4:4 + 6 * 32].view(6, 1, 32)))
    for norm in (False, True):
        x = dict(q=before[:6, :4], k=before[:6, 4:6], norm=True) if norm else {}
        back = lambda **kw: tbe.rotate_heads_backward(q, k, p, f, ws, **(x | kw))  # noqa: E731, B023
        refused(lambda: back(grad_q=wide[1:7, :4]))
        refused(lambda: back(grad_k=wide[:6, 3:5]))
        refused(lambda: back(grad_q=wide[:6, 6:10], grad_k=wide[1:7, 8:10]))
        refused(lambda: back(grad_q=wide[:6, 3:7]))
    refused(lambda: tbe.rotate_heads_backward(before[:6, :4], before[:6, 4:6], p, f, ws, q=q, k=k, norm=True, grad_q=wide[:6, 2:6]))
    refused(lambda: tbe.rotate_heads_backward(before[:6, :4], before[:6, 4:6], p, f, ws, q=q, k=k, norm=True, grad_k=wide[:6, :2]))
    assert torch.equal(wide, before)
    want = tbe.rotate_heads(q, k, p, f)
    got = tbe.rotate_heads(q, k, p, f, q_out=wide[:6, 6:10], k_out=wide[:6, 10:])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    tbe.rotate_heads(q, k, p, f, q_out=wide[1:7, 6:10], k_out=k)
    assert torch.equal(wide[1:7, 6:10], want[0]) and torch.equal(k, want[1]) and torch.equal(wide[:, :4], before[:, :4])
    grads = tbe.rotate_heads_backward(want[0], want[1], p, f, ws, q=before[:6, :4], k=before[:6, 4:6], norm=True)
    over = tbe.rotate_heads_backward(want[0], want[1], p, f, ws, q=q, k=before[:6, 4:6], norm=True, grad_q=q)   # q's gradient over q itself
    assert all(torch.equal(a, b) for a, b in zip(over, grads))


def test_caches_of_one_memory(tbe):
    from paper_2508_03854_amd import Cache
    x, slots = torch.randn(6, 4, 32, device="cuda"), torch.arange(6, device="cuda")
    good = tbe.alloc_cache(6, 4, 32)
    both = torch.zeros(7, 12, 32, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scales = torch.ones(9, 6, device="cuda")
    ks, vs = scales[:4], scales[4:8]
    for k, v in ((both[:6, :4], both[:6, :4]), (both[:6, :4], both[1:, :4]), (both[:6, :4], both[:6, 3:7]), (good.k, good.k), (good.k.view(6, 4, 32), good.k[:6, :4])):
        refused(lambda: tbe.cache_write(Cache(k, v, ks, vs), x, x, slots))
    for a, b in ((ks, ks), (scales[:4], scales[3:7]), (scales.view(-1)[1:25].view(4, 6), scales.view(-1)[24:48].view(4, 6))):
        refused(lambda: tbe.cache_write(Cache(good.k, good.v, a, b), x, x, slots))
    assert not both.view(torch.uint8).any() and not good.k.view(torch.uint8).any() and bool((scales == 1).all())
    tbe.cache_write(good, x, -x, slots)
    beside = Cache(both[:6, 1:5], both[:6, 5:9], ks, vs)
    tbe.cache_write(beside, x, -x, slots)
    assert torch.equal(beside.k.float(), good.k.float()) and torch.equal(beside.v.float(), good.v.float()) and torch.equal(ks, good.k_scales) and torch.equal(vs, good.v_scales)
    # keys that are values too are read
    want = tbe.cache_read(good, slots)[0]
    got = tbe.cache_read(Cache(good.k, good.k, good.k_scales, good.k_scales), slots)
    assert torch.equal(got[0], want) and torch.equal(got[1], want)
    refused(lambda: tbe.cache_read(good, slots, k_out=x, v_out=x))
    wide = torch.zeros(6, 8, 32, device="cuda")
    refused(lambda: tbe.cache_read(good, slots, k_out=wide[:, :4], v_out=wide[:, 3:7]))
    assert not wide.any()
    assert torch.equal(tbe.cache_read(good, slots, k_out=wide[:, :4], v_out=wide[:, 4:])[0], want)
