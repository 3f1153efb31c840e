"""Calls with stream= and without the results' tensors: their memory comes from that stream's pool, so that nothing that is under way on
another stream may still use it, and what is freed goes back there."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def pool_of(t):
    at = t.data_ptr()
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= at < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("no such memory")


def test_results_are_allocated_on_the_stream_that_writes_them():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    tbe = TBE([16, 24], [8, 8])
    dev, s = "cuda", torch.cuda.Stream()
    tables = torch.randn(40 * 8, device=dev)
    ids, bags = torch.randint(0, 16, (12,), device=dev), torch.arange(0, 13, 2, device=dev)
    rows = torch.randn(50, 64, device=dev).to(torch.bfloat16)
    weight, bias = torch.rand(64, device=dev), torch.rand(64, device=dev)
    q, k, v, dout = (torch.randn(50, 2, 32, device=dev).to(torch.bfloat16) for _ in range(4))
    offsets = torch.tensor([0, 20, 50], device=dev)
    table, map_ = torch.randn(2, 4, device=dev), torch.arange(7, dtype=torch.int32, device=dev) % 4
    how = {"bias": table, "bucket_map": map_}
    norm_ws = tbe.alloc_layer_norm_workspace(50, 64)
    spaces = [tbe.alloc_attention_workspace(2, 50, 50, 2, 2, 32, buckets=4, backward=b) for b in (False, True)]

    def all_results(stream):
        y = tbe.layer_norm(rows, weight, bias, stream=stream)
        a = tbe.attention(q, k, v, offsets, offsets, spaces[0], stream=stream, **how)
        return [tbe.forward(tables, ids, bags, 3, stream=stream), tbe.forward_ex(tables, ids, bags, 3, out_dtype=torch.float16, stream=stream), *y, *a,
                *tbe.layer_norm_backward(rows, rows, weight, y[1], y[2], norm_ws, stream=stream),
                *tbe.attention_backward(dout, q, k, v, *a, offsets, offsets, spaces[1], stream=stream, **how)]

    here = all_results(None)
    torch.cuda.synchronize()
    there = all_results(s)
    s.synchronize()
    assert len(there) == 14
    for n, (a, b) in enumerate(zip(here, there)):
        assert torch.equal(a, b), n
        assert pool_of(a) == 0 and pool_of(b) == s.cuda_stream, n
