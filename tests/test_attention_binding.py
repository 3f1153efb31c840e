"""The packed form in which the binding hands over tbe_attention_args has the structure's layout; argument checks that need no GPU."""
import ctypes

from paper_2508_03854_amd import binding as B


def test_packed_arguments_have_the_structures_layout():
    rows = [(101, 7, 8), (102, 9, 10), (103, 11, 12)]
    packed = B._PACK_ATTENTION(1, 2, 3, 4, 5, 6, 1, 0, *rows[0], *rows[1], *rows[2], 201, 202, 203, 1, 0.25, 204, 205, 2, 32, 33)
    assert len(packed) == ctypes.sizeof(B.AttentionArgs)
    a = B.AttentionArgs.from_buffer_copy(packed)
    assert (a.sequences, a.heads, a.kv_heads, a.head_dim, a.q_rows, a.k_rows, a.dtype, a.index_dtype) == (1, 2, 3, 4, 5, 6, 1, 0)
    assert [(r.data, r.row_stride, r.head_stride) for r in (a.q, a.k, a.v)] == rows
    assert (a.q_offsets, a.k_offsets, a.k_lengths, a.causal, a.scale) == (201, 202, 203, 1, 0.25)
    assert (a.bias, a.bucket_map, a.bias_dtype, a.buckets, a.max_distance) == (204, 205, 2, 32, 33)


def test_null_handles_are_refused():
    L = B.load_library()
    a, n = B.AttentionArgs(sequences=1, heads=1, kv_heads=1, head_dim=8), ctypes.c_size_t()
    assert L.tbe_attention_workspace_bytes(None, ctypes.addressof(a), 0, ctypes.byref(n)) == B.EINVAL
    assert L.tbe_attention(None, ctypes.addressof(a), B.Rows(), None, None, 0, None) == B.EINVAL
    assert L.tbe_attention_backward(None, ctypes.addressof(a), B.Rows(), None, B.Rows(), B.Rows(), B.Rows(), B.Rows(), None, None, 0, None) == B.EINVAL
    assert L.tbe_layer_norm(None, None, 0, 0, 0, 8, None, None, 0, 1e-5, None, 0, None, None, None) == B.EINVAL
    assert L.tbe_layer_norm_workspace_bytes(None, 1, 8, ctypes.byref(n)) == B.EINVAL
