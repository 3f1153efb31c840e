"""Results whose heads or rows lie on each other are refused: two writers of one element would leave what the later one wrote."""
import pytest
import torch

from test_gpu_attention import problem, run
from test_gpu_attention_backward import back, upstream

pytestmark = pytest.mark.gpu


def test_results_that_overlap_themselves_are_refused():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE, binding
    tbe = TBE([16], [8])
    p = problem([5, 60], [5, 60], 4, 2, 32, torch.float32)
    dout, fwd = upstream(p), run(tbe, p)
    flat = torch.empty(65 * 128, device="cuda")
    for strides in ((128, 0, 1), (128, 16, 1), (0, 32, 1), (16, 65 * 32, 1)):
        with pytest.raises(binding.TbeError) as e:
            run(tbe, p, out=flat.as_strided((65, 4, 32), strides))
        assert e.value.status == binding.EINVAL, strides
    for name, heads in (("grad_q", 4), ("grad_k", 2), ("grad_v", 2)):
        with pytest.raises(binding.TbeError) as e:
            back(tbe, p, dout, fwd, **{name: flat.as_strided((65, heads, 32), (128, 0, 1))})
        assert e.value.status == binding.EINVAL, name
    # operands may be broadcast, and results lie head by head
    q = p["q"][:, :1].expand(65, 4, 32)
    out = torch.empty(4, 65, 32, device="cuda").transpose(0, 1)
    assert torch.equal(run(tbe, dict(p, q=q), out=out)[0], run(tbe, dict(p, q=q.contiguous()))[0])
