"""More workgroups than one side of a grid can have (2^32 lanes): 2^20 sequences of a few events, 64 heads, forward and both kernels of the
backward, with more keys than queries and the other way round; sampled sequences against the definition."""
import pytest
import torch

import attention_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nk", [(1, 3), (3, 1)])
def test_grids_of_more_than_four_giga_lanes(nq, nk):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    tbe = TBE([16], [8])
    N, H, D = 1 << 20, 64, 8
    g = torch.Generator(device="cuda")
    g.manual_seed(nq)
    q, k, v, dout = (torch.empty(N * n, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for n in (nq, nk, nk, nq))
    qo, ko = (torch.arange(N + 1, dtype=torch.int32, device="cuda") * n for n in (nq, nk))
    ws = tbe.alloc_attention_workspace(N, N * nq, N * nk, H, H, D, backward=True)
    nan = [torch.full_like(x, float("nan")) for x in (q, q, k, v)]
    out, lse = tbe.attention(q, k, v, qo, ko, ws, causal=False, out=nan[0], lse=torch.full((H, N * nq), float("nan"), device="cuda"))
    grads = tbe.attention_backward(dout, q, k, v, out, lse, qo, ko, ws, causal=False, grad_q=nan[1], grad_k=nan[2], grad_v=nan[3])[:3]
    assert not tbe.poll_index_error()
    for s in (0, 1, 31, 32, N // 3, N // 2, N - 33, N - 2, N - 1):
        a, b = slice(s * nq, s * nq + nq), slice(s * nk, s * nk + nk)
        ref = R.reference(q[a], k[b], v[b], [nq], [nk], [0], causal=False, scale=D ** -0.5, dout=dout[a])
        R.check((out[a], lse[:, a], grads[0][a], grads[1][b], grads[2][b]), ref, ("out", "lse", "dq", "dk", "dv"), f"sequence {s}")
    # every row has been written
    assert all(bool(torch.isfinite(t).all()) for t in (lse, out, *grads))
    if nk == 1:
        assert torch.equal(out, v.repeat_interleave(nq, 0))
