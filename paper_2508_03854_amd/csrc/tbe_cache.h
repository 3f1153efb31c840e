// What the kernels on caches of one byte an element share: the caches' rows, and codes as numbers.
#pragma once
#include <hip/hip_runtime.h>

#include "tbe_attention.h"

namespace tbe {

// Codes [rows][heads][dim], a byte each, and scales [heads][rows].
struct CodeRows {
    RowsView codes;
    float* scales;
};

// Four codes as fp32.
template <bool I8>
__device__ __forceinline__ void unpack_codes(const uint32_t w, float* x) {
    if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
    } else {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
    }
}

struct CacheCopyCall {
    tbe_rows rows_of[2];   // keys, values
    CodeRows cache[2];
    const void* slots;
    int64_t rows, cache_rows;
    int heads, dim, io, slots32;
    bool i8;
};
// write: rows into the cache's places; otherwise the places' values into rows
hipError_t launch_cache_copy(const tbe_handle* h, const CacheCopyCall& c, bool write, hipStream_t s);

// attention over such a cache (tbe_cache_attention.hip)
struct CacheAttnPlan {
    int D, pack, block, ranges, qblocks;   // D: elements of a row as the kernels have it; the others: see CacheAttnArgs
    bool own, direct;
    int64_t V;
    size_t spans, part_ml, part_o;   // bytes
};
// light: bfloat16 queries over e4m3; max_pack: heads side by side at most
CacheAttnPlan cache_attn_plan(const AttnShape& sh, bool light, int max_pack = 32);
bool cache_attn_grid_ok(const AttnShape& sh, const CacheAttnPlan& p);   // the launches stay below 2^31 workgroups
size_t cache_attn_workspace(const AttnShape& sh);   // for any max_distance
hipError_t launch_cache_attention(const tbe_handle* h, const AttnArgs& call, const CodeRows (&cache)[2], bool i8, const CacheAttnPlan& p, int io,
                                  void* workspace, hipStream_t s);

}  // namespace tbe
