// Caches of keys and values with one byte an element and a scale for every row and head: rows written into their places, and read back.
//   e4m3  scale 2^e, e the least with max|x| <= 448 2^e (x / scale is then exact before it is rounded to the code's four bits)
//   i8    scale max|x| / 127 rounded to fp32; the code is the whole number nearest to x / scale, exactly
// Bound: the stream, every element read once and written once.  A row's head is in the registers of a few lanes, sixteen elements each, so that
// the codes leave as sixteen bytes a lane; its maximum is found across them.  Measured: 200,003 rows of 8 heads of 128 bfloat16 into places of no order, e4m3:
// 289 us, 4.3 TB/s (the scales, four bytes of a line each, take 23 of them; a copy 5.1 TB/s); 120,011 rows of 8 heads of 96 read back as bfloat16: 132,
// 4.3 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tbe_cache.h"

namespace tbe {

constexpr int kCacheThreads = 256;

// The maximum over the 1, 2, 4 or 8 lanes of a group.
__device__ __forceinline__ uint32_t group_max(uint32_t x, const int lanes) {
    uint32_t o;
    if (lanes >= 2) { o = (uint32_t)dpp_lane_i32<0xB1>((int)x); x = o > x ? o : x; }
    if (lanes >= 4) { o = (uint32_t)dpp_lane_i32<0x4E>((int)x); x = o > x ? o : x; }
    if (lanes >= 8) { o = (uint32_t)dpp_lane_i32<0x141>((int)x); x = o > x ? o : x; }
    return x;
}

// The whole number nearest to x / s (ties to even), |x / s| < 128.  The product with the rounded reciprocal is off by less than one; what it leaves of
// x is exact (a multiple of half of s's last place, below s) and says whether the next number is nearer.
__device__ __forceinline__ int nearest_code(const float x, const float s, const float inv) {
    float q = rintf(x * inv);
    const float left = fmaf(-q, s, x), half = 0.5f * s;
    const bool odd = (int)q & 1;
    if (fabsf(left) > half || (fabsf(left) == half && odd)) q += copysignf(1.f, left);
    return (int)q;
}

struct CacheCopyArgs {
    const char* x[2];          // rows of keys, of values
    int64_t row[2], head[2];   // bytes
    CodeRows cache[2];
    IdxView slots;
    int64_t rows, cache_rows;
    int heads, dim, lanes, beside, per, turns, pieces;   // lanes: of a head, a power of two: its maximum crosses lanes
    uint32_t units;
    int32_t* err;
};

// This lane's place among rows and heads (see copy_shape), and the place of its row in the cache, or -1.
struct CopyPlace {
    int64_t row, slot;
    int head, e;   // first head; first element
};
__device__ __forceinline__ CopyPlace copy_place(const CacheCopyArgs& a, const uint32_t u) {
    const int lane = lane_id(), group = lane / a.lanes, mine = group / a.beside;
    const uint32_t step = u / (uint32_t)a.pieces, piece = u - step * (uint32_t)a.pieces;
    CopyPlace p;
    p.row = mine < a.per ? (int64_t)step * a.per + mine : a.rows;
    p.head = (int)(piece * (uint32_t)(a.turns * a.beside)) + group - mine * a.beside;
    p.e = 16 * (lane - group * a.lanes);
    p.slot = p.row < a.rows ? a.slots[p.row] : -1;
    if (p.slot >= a.cache_rows) {
        *a.err = 1;
        p.slot = -1;
    }
    return p;
}

template <typename T, bool I8>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(const CacheCopyArgs a) {
    constexpr int kN = Frag<T>::kN, kF = 16 / kN;
    const int kv = blockIdx.y;
    const CodeRows cache = a.cache[kv];
    // (all lanes of a wavefront stay in the loop together: the maxima across lanes need them)
    for (uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 6); u < a.units; u += gridDim.x * 4) {
        const CopyPlace p = copy_place(a, u);
        for (int t = 0; t < a.turns; ++t) {
            const int head = p.head + t * a.beside;
            const bool is = p.slot >= 0 && head < a.heads, there = is && p.e < a.dim;
            const T* const from = reinterpret_cast<const T*>(a.x[kv] + (is ? p.row * a.row[kv] + head * a.head[kv] : 0)) + (there ? p.e : 0);
            float x[16];
            uint32_t top = 0;
#pragma unroll
            for (int f = 0; f < kF; ++f) {
                float y[kN];
                Frag<T>::unpack(there ? Frag<T>::load(from + f * kN) : make_uint4(0u, 0u, 0u, 0u), y);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    x[f * kN + i] = y[i];
                    const uint32_t m = __float_as_uint(y[i]) & 0x7FFFFFFFu;   // (as whole numbers NaN is above infinity, that above all others)
                    top = m > top ? m : top;
                }
            }
            top = group_max(top, a.lanes);
            const bool finite = top < 0x7F800000u;
            float scale = 1.f;
            uint32_t code[4];
            if constexpr (I8) {
                if (top > 0u) scale = fmaxf(__uint_as_float(top) / 127.f, 1.17549435e-38f);
                const float inv = 1.f / scale;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    code[w] = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) code[w] |= ((uint32_t)nearest_code(x[4 * w + i], scale, inv) & 0xFFu) << (8 * i);
                }
            } else {
                // 448 = 1.75 * 2^8
                int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
                e = e < -126 ? -126 : e;
                if (top == 0u) e = 0;
                scale = __uint_as_float((uint32_t)(127 + e) << 23);
                const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w] * inv, x[4 * w + 1] * inv, 0, false);
                    c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2] * inv, x[4 * w + 3] * inv, c, true);
                    code[w] = (uint32_t)c;
                }
            }
            if (!is) continue;
            if (there)
                *reinterpret_cast<uint4*>(const_cast<char*>(cache.codes.at(p.slot, head)) + p.e) =
                    finite ? make_uint4(code[0], code[1], code[2], code[3]) : make_uint4(0u, 0u, 0u, 0u);
            if (p.e == 0) cache.scales[(int64_t)head * a.cache_rows + p.slot] = finite ? scale : __builtin_nanf("");
        }
    }
}

template <typename T, bool I8>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(const CacheCopyArgs a) {
    constexpr int kN = Frag<T>::kN, kF = 16 / kN;
    const int kv = blockIdx.y;
    const CodeRows cache = a.cache[kv];
    for (uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 6); u < a.units; u += gridDim.x * 4) {
        const CopyPlace p = copy_place(a, u);
        if (p.row >= a.rows || p.e >= a.dim) continue;
        for (int t = 0; t < a.turns; ++t) {
            const int head = p.head + t * a.beside;
            if (head >= a.heads) continue;
            uint4 c = make_uint4(0u, 0u, 0u, 0u);
            float scale = 0.f;   // (no place: zeros)
            if (p.slot >= 0) {
                c = *reinterpret_cast<const uint4*>(cache.codes.at(p.slot, head) + p.e);
                scale = cache.scales[(int64_t)head * a.cache_rows + p.slot];
            }
            const uint32_t w[4] = {c.x, c.y, c.z, c.w};
            float x[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unpack_codes<I8>(w[i], x + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[4 * i + j] *= scale;
            }
            T* const to = reinterpret_cast<T*>(const_cast<char*>(a.x[kv]) + p.row * a.row[kv] + head * a.head[kv]) + p.e;
#pragma unroll
            for (int f = 0; f < kF; ++f) {
                float y[kN];
#pragma unroll
                for (int i = 0; i < kN; ++i) y[i] = x[f * kN + i];
                Frag<T>::store(to + f * kN, y);
            }
        }
    }
}

template <typename T, bool I8>
static void launch_copy(const CacheCopyArgs& a, const bool write, hipStream_t s) {
    // (A side of a grid has fewer than 2^32 lanes.  At most 4096 workgroups took 297 us where this takes 289, read back 147 / 136.)
    const dim3 grid(std::min((a.units + 3) / 4, 1u << 22), 2);
    if (write) cache_write_kernel<T, I8><<<grid, kCacheThreads, 0, s>>>(a);
    else cache_read_kernel<T, I8><<<grid, kCacheThreads, 0, s>>>(a);
}
template <typename T>
static void launch_code(const CacheCopyArgs& a, const bool write, const bool i8, hipStream_t s) {
    if (i8) launch_copy<T, true>(a, write, s);
    else launch_copy<T, false>(a, write, s);
}

hipError_t launch_cache_copy(const tbe_handle* h, const CacheCopyCall& c, const bool write, hipStream_t s) {
    CacheCopyArgs a{};
    for (int i = 0; i < 2; ++i) {
        const tbe_rows& m = c.rows_of[i];
        const int64_t size = c.io == 0 ? 4 : 2;
        a.x[i] = static_cast<const char*>(m.data);
        a.row[i] = m.row_stride * size;
        a.head[i] = m.head_stride * size;
        a.cache[i] = c.cache[i];
    }
    a.slots = IdxView{c.slots, c.slots32};
    a.rows = c.rows; a.cache_rows = c.cache_rows; a.heads = c.heads; a.dim = c.dim; a.err = h->d_err;
    // A group of lanes has a row's head; heads that are not beside each other come one after the other, unless there would be few wavefronts then.
    // (Reading with 6 lanes for 96 elements, more of them busy but a row's heads in several turns, took 151 us where 8 lanes take 136: 120,011 rows of 8.)
    a.lanes = c.dim / 16;
    while (a.lanes & (a.lanes - 1)) ++a.lanes;
    const HeadShare share = share_heads(64 / a.lanes, c.heads);
    a.beside = share.beside;
    a.per = share.per;
    const int64_t steps = (c.rows + a.per - 1) / a.per, all = (c.heads + a.beside - 1) / a.beside;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(all, 8192 / std::max<int64_t>(1, steps)));
    a.turns = (int)((all + want - 1) / want);
    a.pieces = (int)((all + a.turns - 1) / a.turns);
    a.units = (uint32_t)(steps * a.pieces);
    LaunchTimer tm(h, s, write ? "cache_write" : "cache_read");
    if (c.io == 0) launch_code<float>(a, write, c.i8, s);
    else if (c.io == 1) launch_code<__half>(a, write, c.i8, s);
    else launch_code<bf16_t>(a, write, c.i8, s);
    tm.done();
    return hipGetLastError();
}

}  // namespace tbe
