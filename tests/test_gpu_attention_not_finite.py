"""Attention beside values that are not finite: by the definition, over the pairs that see each other alone, some elements of the
sequence's results are not finite, and the kernels' are so exactly there; all others are, bit by bit, what they are without these values."""
import math

import pytest
import torch

from test_gpu_attention import TYPES, problem, run

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,H,K", [([200, 70], 2, 1), ([500, 330, 600], 2, 1), ([30, 20], 4, 1), ([20, 45] * 3, 2, 2), ([7, 9, 20, 5, 70, 3] * 75, 8, 8)])
def test_values_that_are_hidden_beside_such_that_are_seen(tbe, io, n, H, K):
    """A value that all queries of a sequence see, and one that the later ones see, both not finite, in different elements: either
    reaches the results that see it, and no others."""
    for D in (32, 64, 128):
        for far, buckets in ((0, 0), (20, 8)):
            p = problem(n, n, H, K, D, TYPES[io], buckets=buckets, far=far)
            clean = run(tbe, p)
            for s in (0, 1):
                q0, later = sum(n[:s]), n[s] // 2 + 3
                v = p["v"].clone()
                v[q0, 0, 3], v[q0 + later, 0, 1] = INF, NAN
                got = run(tbe, dict(p, v=v))
                expect = torch.ones_like(clean[0], dtype=torch.bool)
                expect[q0:q0 + n[s], :H // K, 3] = False
                expect[q0 + later:q0 + n[s], :H // K, 1] = False
                assert torch.equal(torch.isfinite(got[0]), expect), (D, far, s, int((torch.isfinite(got[0]) != expect).sum()))
                assert torch.equal(got[0][expect], clean[0][expect]) and torch.equal(got[1], clean[1]), (D, far, s)
