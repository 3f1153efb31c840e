"""Rotation of heads: the packed form of tbe_rotation_args has the structure's layout, the customary frequencies against their formulas, and
argument checks that need no GPU."""
import ctypes
import math

import pytest
import torch

import paper_2508_03854_amd as P
from paper_2508_03854_amd import binding as B


def test_packed_arguments_have_the_structures_layout():
    packed = B._PACK_ROTATION(1, 2, 3, 4, 5, 6, 7, 101, 102, 1, 0.25, 1, 0.5, 103, 104, 2)
    assert len(packed) == ctypes.sizeof(B.RotationArgs)
    a = B.RotationArgs.from_buffer_copy(packed)
    assert (a.q_heads, a.k_heads, a.head_dim, a.rotary_dim, a.rows, a.dtype, a.index_dtype) == (1, 2, 3, 4, 5, 6, 7)
    assert (a.positions, a.frequencies, a.interleaved, a.amplitude, a.norm, a.eps) == (101, 102, 1, 0.25, 1, 0.5)
    assert (a.q_weight, a.k_weight, a.weight_dtype) == (103, 104, 2)


@pytest.mark.parametrize("dim", [2, 4, 10, 64, 256])
def test_frequencies(dim):
    """64-bit functions are off by a few units of 2^-53: 1e-13 of the value."""
    half, base = dim // 2, 5e5
    plain = [base ** (-2 * j / dim) for j in range(half)]

    def close(got, want):
        assert got.dtype == torch.float64 and got.shape == (half,)
        assert all(abs(g - w) <= 1e-13 * w for g, w in zip(got.tolist(), want))

    close(P.rotary_frequencies(dim, base, device="cpu"), plain)
    close(P.rotary_frequencies(dim, base, "linear", 8.0, device="cpu"), [f / 8 for f in plain])
    if dim >= 4:
        got = P.rotary_frequencies(dim, base, "base", 8.0, device="cpu")
        close(got, [(base * 8.0 ** (dim / (dim - 2))) ** (-2 * j / dim) for j in range(half)])
        assert got[0] == 1.0 and abs(got[-1].item() / (plain[-1] / 8) - 1) < 1e-13
    context, lo, hi = 4096.0, 1.0, 32.0
    want = []
    for f in plain:
        turns = context * f / (2 * math.pi)
        kept = min(1.0, max(0.0, (turns - lo) / (hi - lo)))
        want.append(kept * f + (1 - kept) * f / 8)
    close(P.rotary_frequencies(dim, base, "turns", 8.0, context, lo, hi, device="cpu"), want)


def test_frequencies_that_make_no_sense_are_refused():
    f = lambda *a, **k: P.rotary_frequencies(*a, device="cpu", **k)  # noqa: E731
    for args, status in (((0,), B.ESHAPE), ((3,), B.ESHAPE), ((258,), B.ESHAPE), ((2, 1e4, "base", 2.0), B.ESHAPE), ((8, 1.0), B.EINVAL),
                         ((8, math.inf), B.EINVAL), ((8, 1e4, "linear", 0.5), B.EINVAL), ((8, 1e4, "linear", math.nan), B.EINVAL),
                         ((8, 1e4, "turns", 2.0, 0.0), B.EINVAL), ((8, 1e4, "turns", 2.0, 100.0, 4.0, 4.0), B.EINVAL),
                         ((8, 1e4, "turns", 2.0, 100.0, -1.0, 4.0), B.EINVAL), ((8, 1e300, "base", 1e300), B.EINVAL)):
        with pytest.raises(P.TbeError) as e:
            f(*args)
        assert e.value.status == status, args
    with pytest.raises(KeyError):
        f(8, 1e4, "other")
    assert B.load_library().tbe_rotary_frequencies(8, 1e4, 9, 1.0, 0.0, 0.0, 0.0, None) == B.EDTYPE
    assert B.load_library().tbe_rotary_frequencies(8, 1e4, 0, 1.0, 0.0, 0.0, 0.0, None) == B.EINVAL


def test_null_handles_are_refused():
    L = B.load_library()
    a, n = B.RotationArgs(q_heads=1, head_dim=8), ctypes.c_size_t()
    at, r = ctypes.addressof(a), B.Rows()
    assert L.tbe_rotate_workspace_bytes(None, at, ctypes.byref(n)) == B.EINVAL
    assert L.tbe_rotate_heads(None, at, r, r, r, r, None) == B.EINVAL
    assert L.tbe_rotate_heads_backward(None, at, r, r, r, r, r, r, None, None, None, 0, None) == B.EINVAL
