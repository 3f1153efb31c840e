"""Caches of one byte an element: the packed form of tbe_cache has the structure's layout; argument checks that need no GPU."""
import ctypes

from paper_2508_03854_amd import binding as B


def test_packed_cache_has_the_structures_layout():
    packed = B._PACK_CACHE(1, 2, 3, 1, 101, 4, 5, 102, 6, 7, 103, 104)
    assert len(packed) == ctypes.sizeof(B.CacheArgs)
    c = B.CacheArgs.from_buffer_copy(packed)
    assert (c.rows, c.heads, c.head_dim, c.code, c.k_scales, c.v_scales) == (1, 2, 3, 1, 103, 104)
    assert [(r.data, r.row_stride, r.head_stride) for r in (c.k, c.v)] == [(101, 4, 5), (102, 6, 7)]


def test_null_handles_are_refused():
    L = B.load_library()
    a, c, n = B.AttentionArgs(sequences=1, heads=1, kv_heads=1, head_dim=16), B.CacheArgs(heads=1, head_dim=16), ctypes.c_size_t()
    at, ct, r = ctypes.addressof(a), ctypes.addressof(c), B.Rows()
    assert L.tbe_cache_write(None, ct, r, r, 0, None, 0, 0, None) == B.EINVAL
    assert L.tbe_cache_read(None, ct, None, 0, 0, r, r, 0, None) == B.EINVAL
    assert L.tbe_cache_attention_workspace_bytes(None, at, ctypes.byref(n)) == B.EINVAL
    assert L.tbe_cache_attention(None, at, ct, r, None, None, 0, None) == B.EINVAL
