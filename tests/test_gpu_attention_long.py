"""Attention and its gradients where the average length lies on either side of what a workgroup of shared tiles begins at: against the
definition in 64 bits (tests/attention_reference.py derives the bounds), with one-row and empty sequences among the long ones."""
import math

import pytest
import torch

import attention_reference as R
from test_gpu_attention import TYPES, problem, run
from test_gpu_attention_short import both

pytestmark = pytest.mark.gpu

LONG = [900, 1, 0, 513, 640, 129, 255]          # 348 on average
MIDDLE = [200, 1, 0, 161, 260, 96, 255, 130]    # 138
MANY = [150, 90, 0, 129, 64, 1, 200, 33] * 9    # 83, in more wavefronts of 32 rows than make neighbours share one


@pytest.fixture(scope="module")
def tbe():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2508_03854_amd import TBE
    return TBE([16], [8])


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_long_and_middling_sequences(tbe, io, D):
    for n, H, K in ((LONG, 2, 1), (MIDDLE, 2, 2), (MANY, 8, 4)):
        for causal, buckets, far in ((True, 16, 60), (False, 9, 200), (True, 0, 0)):
            both(tbe, problem(n, n, H, K, D, TYPES[io], causal=causal, buckets=buckets, far=far), f"{io} {D} {len(n)} {causal} {buckets}")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_other_numbers_of_keys(tbe, io):
    for D in (32, 64, 128):
        for nq, nk in ((LONG, [n // 3 + 5 for n in LONG]), ([n // 2 for n in LONG], LONG), ([n // 3 for n in LONG], LONG), (MIDDLE, [3 * n for n in MIDDLE])):
            both(tbe, problem(nq, nk, 2, 1, D, TYPES[io], buckets=16, far=100), f"{io} {D} {sum(nq)} {sum(nk)}")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_far_tables(tbe, io):
    """A group of heads whose tables of distances do not fit beside each other: keys share tiles however few they are."""
    for D, n in ((64, LONG), (128, MIDDLE), (128, LONG)):
        both(tbe, problem(n, n, 4, 1, D, TYPES[io], buckets=32, far=1024), f"{io} {D} {len(n)}")


@pytest.mark.parametrize("io", ["f32", "f16", "bf16"])
def test_values_that_are_not_finite_reach_only_who_sees_them(tbe, io):
    for D in (32, 64, 128):
        for n in ([500, 330], [150, 190]):
            p = problem(n, n, 2, 1, D, TYPES[io])
            clean = run(tbe, p)[0]
            at = [min(n[0] - 1, 301), 140]      # a key of either sequence
            p["v"][p["k0"][0] + at[0], 0, 3] = math.inf
            p["v"][p["k0"][1] + at[1], 0, 1] = float("nan")
            got = run(tbe, p)[0]
            expect = clean.clone()
            expect[at[0]:n[0], :, 3] = math.inf
            expect[n[0] + at[1]:, :, 1] = float("nan")
            seen = torch.isfinite(expect)
            assert torch.equal(torch.isnan(got), torch.isnan(expect)) and torch.equal(got == math.inf, expect == math.inf), (D, n)
            assert (got[seen].double() - clean[seen].double()).abs().max() <= 4 * (R.T[TYPES[io]] + 600 * R.U) * clean[seen].abs().max().double()
