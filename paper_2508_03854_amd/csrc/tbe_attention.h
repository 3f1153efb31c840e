// What the attention kernels share: the sequences' places, tiles of rows in LDS, matrix products of 32 x 32 tiles.
//
// Lanes and tiles.  A product of the matrix cores leaves a 32 x 32 tile with one column per lane: lane l holds column l % 32 and, of the
// 32 rows, those 8 i + 4 (l / 32) + e  (i, e < 4) in register 4 i + e.  The kernels put what a softmax runs over into the rows and what
// it is one of into the columns, so that row maxima and sums are a lane's own, but for one exchange between the wavefront's halves,
// and the tile of probabilities is, as it lies in the registers, an operand of the next product (fragment m: registers 8 m .. 8 m + 7
// of a 16-bit type, 4 m .. 4 m + 3 of fp32).  The other operand's fragments then take their rows in the same order.
#pragma once
#include <hip/hip_runtime.h>

#include "tbe_elems.h"
#include "tbe_internal.h"

namespace tbe {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

// x, as a value that the compiler does not know: what is computed from it is computed again, not kept in registers through the loops in between
__device__ __forceinline__ int anew(int x) {
    asm volatile("" : "+v"(x));
    return x;
}
// a value that all lanes hold, as a scalar
__device__ __forceinline__ int uniform(const int x) { return __builtin_amdgcn_readfirstlane(x); }

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kTabMargin = 68;         // a tile that reaches into the table of distances reaches at most 66 beyond its ends
// So many wavefronts, were there one for every 32 rows of a sequence and head, and short sequences share wavefronts.  A wavefront of one sequence /
// shared ones, 8 heads of 64 bfloat16, lengths lognormal (7 in the middle, 12 on average), us: 256 sequences (2816 wavefronts) forward 18.1 / 13.2,
// dq 32.8 / 24.2; 1024 (11264) 45.6 / 23.4, 78.7 / 45.7; 4096 156 / 64, 265 / 121; for 64 (704), on their own 11.1 and 20.4.
constexpr int64_t kManyUnits = 2048;
constexpr int kTabBytes = 24 << 10;    // LDS for such tables

// Sequences of few rows have a wavefront for every 32 of them, longer ones a workgroup for every 128, which share the tiles of the other side: up
// to 64 rows on average, and as long as neither side has more than `most`.  Shared / on their own, us, as many sequences as named of that
// length, with bias, causal:
//   forward  32 bfloat16: 512 of 128 46 / 26, of 180 54 / 43, 256 of 150 with 300 keys 38 / 39, 64 of 400 23 / 22
//            64 bfloat16: 512 of 80 76 / 49, of 128 149 / 82, of 180 189 / 154, 64 of 256 33 / 30, of 600 79 / 97;  fp32: 64 of 256 66 / 60
//            128 bfloat16: 64 of 80 15.0 / 14.3, of 128 17.6 / 25.1;  fp32: 64 of 128 33 / 44
//   dq       32 bfloat16: 512 of 128 113 / 87, of 180 144 / 135;  fp32: 512 of 128 303 / 235, of 200 415 / 419
//            64 bfloat16: 512 of 128 381 / 200, of 180 483 / 304, 64 of 256 81 / 63, 256 of 245 266 / 234;  fp32: 512 of 128 671 / 292,
//            64 of 400 258 / 196, of 600 384 / 345
//            128 bfloat16: 64 of 128 36 / 46;  fp32: 69 / 81
//   dk, dv   32 bfloat16: 512 of 128 69 / 39, of 180 72 / 62
//            64 bfloat16: 512 of 128 252 / 157, 64 of 180 41 / 34, of 256 47 / 47;  fp32: 64 of 400 300 / 190, of 600 404 / 353
//            128 bfloat16: 64 of 128 40 / 31, of 400 141 / 99, 16 of 2000 345 / 333, 4 of 4000 478 / 257 (the shared kernel has one
//            wavefront a SIMD, which waits at its barriers);  fp32: 64 of 80 44 / 50, of 200 126 / 156
inline bool attn_few(const int64_t mean, const int64_t other, const int64_t most) { return mean <= 64 || (mean <= most && other <= most); }

// Sixteen zero bytes: what stands behind a sequence's end, or behind a row's, is read from here.
static __device__ const uint4 attn_zeros = {0u, 0u, 0u, 0u};

template <typename T>
struct Mma {   // 16-bit types: fragments of 8 elements a lane, 16 of the summed axis at a time
    static constexpr int kE = 8, kK = 16, kDown = 2, kMfmas = 1;   // kDown: LDS reads of a fragment down the rows; kMfmas: of its product
    static __device__ __forceinline__ f32x16_t mma(const uint4 a, const uint4 b, const f32x16_t c) {
        if constexpr (__is_same(T, bf16_t))
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
        else
            return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
    // registers 8 m .. 8 m + 7 of a tile as an operand; each is rounded once.  (As numbers of fp32: where a product is next rounded to binary16, the
    // compiler does both at once in one copy of a loop and not in another, and the two would differ.)
    static __device__ __forceinline__ uint4 pack(f32x16_t s, const int m) {
        const T* const t = nullptr;
        if constexpr (__is_same(T, __half)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = s[8 * m + i];
                asm("" : "+v"(x));
                s[8 * m + i] = x;
            }
        }
        return make_uint4(pack2(t, s[8 * m], s[8 * m + 1]), pack2(t, s[8 * m + 2], s[8 * m + 3]), pack2(t, s[8 * m + 4], s[8 * m + 5]),
                          pack2(t, s[8 * m + 6], s[8 * m + 7]));
    }
};
template <>
struct Mma<float> {   // four products of two of the summed axis each
    static constexpr int kE = 4, kK = 8, kDown = 4, kMfmas = 4;
    static __device__ __forceinline__ f32x16_t mma(const uint4 a, const uint4 b, f32x16_t c) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint4 pack(const f32x16_t& s, const int m) {
        return make_uint4(__float_as_uint(s[4 * m]), __float_as_uint(s[4 * m + 1]), __float_as_uint(s[4 * m + 2]), __float_as_uint(s[4 * m + 3]));
    }
};

// whether an element of a result is not finite
template <int N>
__device__ __forceinline__ bool not_finite(const f32x16_t (&o)[N]) {
    float test = 0.f;   // stays 0, or becomes NaN
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) test = fmaf(o[d][r], 0.f, test);
    return test != 0.f;
}

// The fragments of one column's row of D elements, dim of them there; `is` false: zeros (the row is one that can be read all the same).
// Without a branch between the lanes: where registers are short, the compiler was seen to place copies of registers that live on at the head of the
// block behind such a branch, before the lanes that were off come back (ROCm 7.2).  These lanes lost the values, and a gradient of the bias came
// out wrong now and then.  So nothing that the tiles' loops are reached through, or that runs within them, lets lanes go different ways.
template <typename T, int D>
__device__ __forceinline__ void column_row(uint4 (&f)[D / Mma<T>::kK], const char* row, const bool is, const int half, const int dim) {
    constexpr int kE = Mma<T>::kE, kK = Mma<T>::kK;
    if (dim == D) {
#pragma unroll
        for (int c = 0; c < D / kK; ++c) f[c] = *reinterpret_cast<const uint4*>(row + (kK * c + kE * half) * sizeof(T));
    } else {
#pragma unroll
        for (int c = 0; c < D / kK; ++c) {
            const int e = kK * c + kE * half;
            f[c] = *reinterpret_cast<const uint4*>(row + (e < dim ? e : 0) * sizeof(T));
        }
    }
#pragma unroll
    for (int c = 0; c < D / kK; ++c) {
        const bool there = is && kK * c + kE * half < dim;
        f[c] = make_uint4(there ? f[c].x : 0u, there ? f[c].y : 0u, there ? f[c].z : 0u, there ? f[c].w : 0u);
    }
}
// the sign of the scale
template <typename T, int N>
__device__ __forceinline__ void flip_signs(uint4 (&f)[N]) {
    constexpr uint32_t sign = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
#pragma unroll
    for (int c = 0; c < N; ++c) f[c] = make_uint4(f[c].x ^ sign, f[c].y ^ sign, f[c].z ^ sign, f[c].w ^ sign);
}

// whether a lane of those that share tiles says so: of the workgroup's four wavefronts (SHARE = 4, all of them here; votes: LDS that is used for
// nothing else), or of this one
template <int SHARE>
__device__ __forceinline__ bool any_sharer(const bool here, int* votes, const int wave) {
    bool any = __any(here);
    if constexpr (SHARE == 4) {
        if (lane_id() == 0) votes[wave] = any;
        __syncthreads();
        any = uniform(votes[0] | votes[1] | votes[2] | votes[3]) != 0;
    }
    return any;
}
// every lane's BYTES bytes to LDS, one lane's behind the other's
template <int BYTES>
__device__ __forceinline__ void load_lds(const void* from, void* to) {
    const auto src = (const __attribute__((address_space(1))) void*)from;
    const auto dst = (__attribute__((address_space(3))) void*)to;
    if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds(src, dst, 16, 0, 0);
    else __builtin_amdgcn_global_load_lds(src, dst, 4, 0, 0);
}

// Ends a run of matrix products whose results are next read on the other side of a branch.  A result may be read by a vector instruction only
// 11 (16-bit types) or 18 (fp32) issue slots after its product; the hardware does not wait, and the compiler, which has to fill in
// the slots, was seen to count them along one of the branch's two ways only (7 slots on the other, and results of the last product but
// partly there).
template <typename T>
__device__ __forceinline__ void settle() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15");
    if constexpr (sizeof(T) == 4) asm volatile("s_nop 3");
    __builtin_amdgcn_sched_barrier(0);
}

// How a run of N products of fragments from LDS is to be put in order: the reads of AHEAD fragments under way before the first product, then
// a product for every further fragment.  READS, MFMAS: instructions of a fragment.
template <int N, int READS, int MFMAS, int AHEAD>
__device__ __forceinline__ void reads_ahead() {
    constexpr int kAhead = AHEAD < N ? AHEAD : N;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
    for (int i = 0; i < N - kAhead; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, MFMAS, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) __builtin_amdgcn_sched_group_barrier(0x008, MFMAS, 0);
}

// A tile of rows of D elements in LDS, sixteen-byte chunks: chunk c of row r lies at place c ^ swizzle(r) of its row.  The LDS serves 256
// bytes a clock: of 16-byte reads along the rows those of 16 rows, which therefore lie in 16 different chunks of the 64 banks; of 8-byte
// reads down the rows those of 4 rows by 4 chunks, which therefore lie in different quarters.  (The row's number alone as the swizzle
// left the latter four to a quarter, 60 % of the LDS's clocks.)  Rows arrive straight from memory; a wavefront's 64 chunks land one
// behind the other, so it is the source that is permuted.
template <typename T, int D>
struct Tile {
    static constexpr int kChunks = D * (int)sizeof(T) / 16;   // of a row: 4 to 32
    static constexpr uint32_t kLower = sizeof(T) == 4 ? 0x7F800000u : (__is_same(T, bf16_t) ? 0x7F80u : 0x7C00u);   // an exponent of all ones
    static __device__ __forceinline__ int swizzle(const int r) {
        return kChunks == 4 ? (r >> 2) & 3 : (kChunks == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3));
    }
    // fragment c of the tile's row r, along the row (the lanes' halves take alternate chunks)
    static __device__ __forceinline__ uint4 along(const char* lds, const int r, const int c, const int half) {
        return *reinterpret_cast<const uint4*>(lds + (r * kChunks + ((2 * c + half) ^ swizzle(r))) * 16);
    }
    // fragment m down the rows first + ..., column 32 t + l % 32: the rows that registers of fragment m stand for
    static __device__ __forceinline__ uint4 down(const char* lds, const int first, const int m, const int t, const int l = lane_id()) {
        const int half = l >> 5;
        if constexpr (sizeof(T) == 2) {
            // sixteen lanes read four rows of sixteen columns, and get a column of four rows each
            typedef __attribute__((address_space(3))) s16x4_t* lds_ptr;
            const int j = l & 15, c = 4 * t + 2 * ((l >> 4) & 1) + ((j & 3) >> 1), r = first + 16 * m + 4 * half + (j >> 2);
            const char* const p = lds + (r * kChunks + (c ^ swizzle(r))) * 16 + (j & 1) * 8;
            const char* const q = lds + ((r + 8) * kChunks + (c ^ swizzle(r + 8))) * 16 + (j & 1) * 8;
            const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p));
            const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)q));
            return make_uint4(a.x, a.y, b.x, b.y);
        } else {
            const int e = 32 * t + (l & 31), r = first + 8 * m + 4 * half;
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = *reinterpret_cast<const uint32_t*>(lds + ((r + i) * kChunks + ((e >> 2) ^ swizzle(r + i))) * 16 + (e & 3) * 4);
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    // What a column does not see has the factor 0, but 0 times an element that is not finite is not 0.  Where a product's results are not finite
    // though not all is seen, it is taken once more, of fragments without such elements (cleaned), and the elements themselves are multiplied
    // one by one for those columns that see them (add_not_finite): the other columns' results are, bit by bit, as if these were not there.
    static __device__ __forceinline__ uint4 cleaned(const uint4 v) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = (w[i] & kLower) == kLower ? w[i] & (sizeof(T) == 4 ? 0u : 0xFFFF0000u) : w[i];
            w[i] = sizeof(T) == 2 && (w[i] >> 16 & kLower) == kLower ? w[i] & 0xFFFFu : w[i];
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the rows first .. first + 31 with an element that is not finite, a bit each
    static __device__ __forceinline__ uint32_t not_finite(const char* lds, const int first, const int l) {
        uint32_t rows = 0;
#pragma unroll 1
        for (int i = 0; i < 32 * kChunks; i += 64) {
            const int n = i + l;
            const uint4 v = *reinterpret_cast<const uint4*>(lds + (first * kChunks + n) * 16), c = cleaned(v);
            rows |= (v.x ^ c.x) | (v.y ^ c.y) | (v.z ^ c.z) | (v.w ^ c.w) ? 1u << (n / kChunks) : 0u;
        }
#pragma unroll
        for (int i = 32; i; i >>= 1) rows |= __shfl_xor(rows, i);
        return (uint32_t)uniform((int)rows);
    }
    // o += x times the elements that are not finite of rows first .. first + 31, for the columns that see them: column l % 32 the rows first + lo ..
    // first + end - 1
    static __device__ __forceinline__ void add_not_finite(f32x16_t (&o)[D / 32], const char* lds, const int first, const f32x16_t& x, const int lo, const int end, const int l) {
        const int col = l & 31, half = l >> 5;
#pragma unroll 1
        for (uint32_t rows = not_finite(lds, first, l); rows; rows &= rows - 1) {
            const int j = __ffs(rows) - 1, r = first + j;
            float by = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) by = 4 * (j >> 3) + (j & 3) == i ? x[i] : by;
            by = __shfl(by, col + 8 * (j & 4));
            const bool sees = j >= lo && j < end;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    __builtin_amdgcn_sched_barrier(0);
                    const char* const p = lds + r * kChunks * 16;
                    float e[4];
                    if constexpr (sizeof(T) == 4) {
                        const float4 v = *reinterpret_cast<const float4*>(p + ((8 * d + 2 * i + half) ^ swizzle(r)) * 16);
                        e[0] = v.x; e[1] = v.y; e[2] = v.z; e[3] = v.w;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(p + ((4 * d + i) ^ swizzle(r)) * 16 + 8 * half);
                        float both[8];
                        Frag<T>::unpack(make_uint4(v.x, v.y, 0u, 0u), both);
                        e[0] = both[0]; e[1] = both[1]; e[2] = both[2]; e[3] = both[3];
                    }
#pragma unroll
                    for (int n = 0; n < 4; ++n)
                        o[d][4 * i + n] = fmaf(by, sees && !(fabsf(e[n]) < __builtin_inff()) ? e[n] : 0.f, o[d][4 * i + n]);
                }
        }
    }
    // ROWS rows from row j0 of a sequence on, of which there are `rows`, by WAVES wavefronts (this one is number w); complete after
    // loads_done().  `stride`: bytes from row to row
    template <int ROWS, int WAVES>
    static __device__ __forceinline__ void fetch(char* lds, const char* base, const int64_t stride, const int j0, const int rows, const int dim, const int w,
                                                 const int l = lane_id()) {
        constexpr int kLoads = ROWS * kChunks / 64 / WAVES;
        static_assert(kLoads * 64 * WAVES == ROWS * kChunks, "whole loads");
        const char* const from = base + (int64_t)j0 * stride;
        if (j0 + ROWS <= rows && dim == D) {   // (offsets that stay the same from tile to tile)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int n = (w * kLoads + i) * 64 + l, r = n / kChunks, c = (n % kChunks) ^ swizzle(r);
                load_lds<16>(from + (uint32_t)(r * (uint32_t)stride + c * 16), lds + (w * kLoads + i) * 1024);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int n = (w * kLoads + i) * 64 + l, r = n / kChunks, c = (n % kChunks) ^ swizzle(r);
                const bool there = j0 + r < rows && c * 16 < dim * (int)sizeof(T);
                load_lds<16>(there ? from + (uint32_t)(r * (uint32_t)stride + c * 16) : reinterpret_cast<const char*>(&attn_zeros), lds + (w * kLoads + i) * 1024);
            }
        }
    }
};
// waits for this wavefront's loads (vmcnt 0, the other counters as they are); as a builtin, so that the compiler knows of it
__device__ __forceinline__ void loads_done() {
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// x's value in the lane 32 further on (or back), combined with this lane's
__device__ __forceinline__ float halves_max(const float x) {
    const unsigned u = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Wide rows: beyond this, one fp32 number for lse (here as an exponent of 2) has too few bits left for the logarithm of the sum, which moves all
// probabilities of the row by up to 2^-23 |lse|: 8e-6 of themselves in fp32, 6e-5 in types that are rounded to 2^-9 or 2^-12.
template <typename T>
__device__ __forceinline__ bool wide_row(const float lse2) {
    return fabsf(lse2) > (sizeof(T) == 4 ? 64.f : 512.f) && lse2 < __builtin_inff();
}

// A matrix [rows][heads][dim]: bytes from row to row and from head to head.
struct RowsView {
    const char* p;
    int64_t row, head;
    __device__ __forceinline__ const char* at(const int64_t r, const int h) const { return p + r * row + h * head; }
};

struct AttnArgs {
    RowsView q, k, v, o, dout, dq, dk, dv;
    float* lse;               // [H][q_rows]
    // [H][q_rows] of the backward: row sums of P dP; a row's probabilities are weight 2^(x - lse2), where lse2 is +infinity for rows that saw
    // nothing and weight 1 for all but wide rows
    float *delta, *lse2, *weight;
    IdxView q_off, k_off, k_len;   // k_len.p may be null
    int N, H, kv, group, dim, causal;
    int64_t q_rows, k_rows;
    float scale, scale2;      // scale2: |scale| log2(e); negative: scale < 0
    int negative;
    const void* bias;         // [H][buckets]
    int bias_io, buckets, far;
    const int32_t* map;
    int32_t* err;
    // how queries are shared out: a unit has `pack` heads of a group side by side and qpt queries of each per 32 columns
    int pack, qpt, block, V, splits;   // block: queries of a unit; V: units of a head that the sequences may need; splits of the keys
    int together;             // the wavefronts of a workgroup take parts of one split's keys and join them
    float *part_o, *part_ml;
    float* part_bias;
};

// Sequence of unit v of V = q_rows / block + N: sequence s owns units offsets[s] / block + s on, as many as it needs, and there is
// always room (a sequence never needs more than its rows / block, rounded down, and one).  All lanes of a wavefront together, 64 offsets
// at a time.
__device__ __forceinline__ int find_sequence(const IdxView off, const int N, const uint32_t v, const uint32_t block) {
    int lo = 0, hi = N;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, s = lo + lane_id() * step;
        const bool before = s < hi && (uint32_t)off[s] / block + (uint32_t)s <= v;
        const uint64_t m = __ballot(before);
        const int k = m ? 63 - __builtin_clzll(m) : 0;
        lo += k * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    return uniform(lo);
}

// The largest s below N with offsets[s] <= row: the sequence of a row, if offsets[s + 1] > row.
__device__ __forceinline__ int find_row(const IdxView off, const int N, const int64_t row) {
    int lo = 0, hi = N;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, s = lo + lane_id() * step;
        const uint64_t m = __ballot(s < hi && off[s] <= row);
        const int k = m ? 63 - __builtin_clzll(m) : 0;
        lo += k * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    return uniform(lo);
}
// ... of each of 32 neighbouring rows, for the lane l % 32 that has it (rows: there are so many in all).  The ends of the next 64 sequences are
// loaded together, and every lane counts those that lie before its row; where many sequences are empty, 64 more.
__device__ __forceinline__ int lane_sequence(const IdxView off, const int N, const int64_t row0, const int64_t rows) {
    const int64_t row = row0 + (lane_id() & 31);
    int base = find_row(off, N, row0), mine = base;
    bool open = row < rows;
    while (__any(open)) {
        const int s = base + 1 + lane_id();
        const int64_t e = s <= N ? off[s] : INT64_MAX;
        const int end = e > row0 + 32 ? 32 : (int)(e - row0 < 0 ? 0 : e - row0);   // rows of the 32 before it
        int n = 0;   // ends at or before this lane's row; they ascend
#pragma unroll
        for (int step = 32; step; step >>= 1)
            if (__shfl(end, n + step - 1) <= (int)(row - row0)) n += step;
        n += n == 63 && __shfl(end, 63) <= (int)(row - row0);
        if (open) mine = base + n;
        open = open && n == 64 && base + 64 < N;
        base += 64;
    }
    return mine < N ? mine : N - 1;
}

struct Sequence {
    int64_t q0, k0;   // first rows
    int nq, nk;       // queries, keys
    int cap;          // rows of k and v that are the sequence's, filled or not
};
// The five numbers of a sequence, one in each of the first lanes: one trip to memory.
__device__ __forceinline__ int64_t sequence_numbers(const AttnArgs& a, const int s) {
    const int l = lane_id();
    const IdxView& from = l < 2 ? a.q_off : (l < 4 || !a.k_len.p ? a.k_off : a.k_len);
    return l < 5 ? from[s + (l < 4 ? l & 1 : 0)] : 0;
}
// false: they are not what they have to be (reported)
__device__ __forceinline__ bool take_sequence(const AttnArgs& a, const int s, const int64_t mine, Sequence& q) {
    const int64_t q0 = lane_i64(mine, 0), q1 = lane_i64(mine, 1), k0 = lane_i64(mine, 2), k1 = lane_i64(mine, 3);
    const int64_t n = a.k_len.p ? lane_i64(mine, 4) : k1 - k0;
    bool ok = q0 >= 0 && q0 <= q1 && q1 <= a.q_rows && k0 >= 0 && k0 <= k1 && k1 <= a.k_rows && n >= 0 && n <= k1 - k0;
    if (s == 0) ok = ok && q0 == 0 && k0 == 0;
    if (s == a.N - 1) ok = ok && q1 == a.q_rows && k1 == a.k_rows;
    q.q0 = q0; q.k0 = k0;
    q.nq = uniform((int)(q1 - q0)); q.nk = uniform((int)n); q.cap = uniform((int)(k1 - k0));
    if (!ok && lane_id() == 0) *a.err = 1;
    return ok;
}
// A lane's own sequence, where the rows of several share a tile.
struct LaneSequence {
    int64_t q0, q1, k0, k1;
    bool fits;
};
__device__ __forceinline__ LaneSequence lane_numbers(const AttnArgs& a, const int s) {
    LaneSequence q;
    q.q0 = a.q_off[s]; q.q1 = a.q_off[s + 1]; q.k0 = a.k_off[s]; q.k1 = a.k_off[s + 1];
    q.fits = q.q0 >= 0 && q.q0 <= q.q1 && q.q1 <= a.q_rows && q.k0 >= 0 && q.k0 <= q.k1 && q.k1 <= a.k_rows;
    if (s == 0) q.fits = q.fits && q.q0 == 0 && q.k0 == 0;
    if (s == a.N - 1) q.fits = q.fits && q.q1 == a.q_rows && q.k1 == a.k_rows;
    if (!q.fits) *a.err = 1;
    return q;
}
// All sequences looked over by `units` wavefronts, 64 at a time.
__device__ __forceinline__ void judge_all(const AttnArgs& a, const uint32_t unit, const uint32_t units) {
    for (int64_t s = (int64_t)unit * 64 + lane_id(); s < a.N; s += (int64_t)units * 64) (void)lane_numbers(a, (int)s);
}
__device__ __forceinline__ int wave_min_i32(const int x) { return -wave_max_i32(-x); }

// Offsets that do not ascend may keep the search from ever meeting the sequence that is wrong, so that unit n of the first head (there are
// at least as many as sequences) looks at sequence n besides: `peek` is loaded early and judged when the unit is done.
__device__ __forceinline__ void judge(const AttnArgs& a, const bool looks, const int n, const int64_t peek) {
    Sequence q;
    if (looks) (void)take_sequence(a, n, peek, q);
}

// The bias of a head by (key's place - query's place), as an exponent of 2: entry far + kTabMargin + (key - query), distances beyond
// `far` like `far` itself.  A finite bias beyond +-1e30 counts as that (so that it stays finite here); a bucket outside the table
// counts as no bias and is reported.
__device__ __forceinline__ int tab_size(const int far) { return 2 * far + 1 + 2 * kTabMargin; }
__device__ __forceinline__ void fill_bias(float* tab, const AttnArgs& a, const int head0, const int heads, const int threads,
                                          uint16_t* bucket = nullptr) {
    const int size = tab_size(a.far), used = a.causal ? a.far + kTabMargin + 1 : size;
    for (int n = threadIdx.x; n < heads * used; n += threads) {
        const int g = n / used, t = n - g * used;
        int d = a.far + kTabMargin - t;   // query - key
        d = d > a.far ? a.far : (d < -a.far ? -a.far : d);
        const int b = a.map[d + a.far];
        float x = 0.f;
        if ((uint32_t)b < (uint32_t)a.buckets) {
            x = param_load(a.bias, a.bias_io, (int64_t)(head0 + g) * a.buckets + b);
            if (x > 1e30f && x < __builtin_inff()) x = 1e30f;
            if (x < -1e30f && x > -__builtin_inff()) x = -1e30f;
            x *= kLog2e;
        } else {
            *a.err = 1;
        }
        tab[g * size + t] = x;
        if (bucket) bucket[t] = (uint16_t)((uint32_t)b < (uint32_t)a.buckets ? b : 0xFFFF);
    }
}

// Workgroups are dealt to the 8 dies one by one; each die takes a run of neighbours, so that those that read the same keys share its
// level-2 cache: 2 sequences of 6000, 16 heads of 128 over 4 bfloat16, forward in the order of the grid 440 us, in this one 393; 48 sequences with
// 61 queries each, 8 heads of 64, 81 / 63; 4 of 2500, 8 heads of 64 over 2, dq 154 / 129, dk and dv 147 / 119.  n or more: nothing to do.
__device__ __forceinline__ uint32_t die_order(const uint32_t n) {
    const uint32_t wg = blockIdx.y * gridDim.x + blockIdx.x, run = (n + 7u) / 8u;
    return (wg >> 3) < run ? (wg & 7u) * run + (wg >> 3) : n;
}
// The grid for it: a side of a grid has fewer than 2^32 lanes, which 2^20 sequences of a few events with 64 heads exceed.
inline dim3 die_grid(const uint64_t n) {
    const uint64_t all = (n + 7) / 8 * 8, side = (uint64_t)1 << 22;
    return all <= side ? dim3((unsigned)all) : dim3((unsigned)side, (unsigned)((all + side - 1) / side));
}
// A workgroup's head (or heads) and which of the head's items it has: one head after the other, which keeps the keys of few heads in the cache; short
// sequences (SHARE = 0), whose wavefronts wait for memory first of all, one item after the other, so that heads that lie in the same cache
// lines are read together: 4096 sequences of 12 events on average, 4 heads of 32 bfloat16, head after head / item after item, us: forward 30.8 /
// 22.4, dq 71 / 59, dk and dv 46 / 41; 512 of 128, 8 heads of 64, forward 86 / 84.
template <int SHARE>
__device__ __forceinline__ void head_and_item(const uint32_t wg, const uint32_t per_head, const uint32_t heads, int& head, uint32_t& item) {
    constexpr bool beside = SHARE == 0;
    const uint32_t by = beside ? heads : per_head, d = wg / by, m = wg - d * by;
    head = uniform(beside ? m : d);
    item = uniform(beside ? d : m);
}

}  // namespace tbe
