// Attention over a cache of one byte an element (see tbe355.h): the keys' and values' codes are multiplied as they are, their scales where the scores and
// probabilities are in fp32 anyway; no value of the cache is ever written out.
//   S^T = C_k Q^T  (a tile: 32 keys x 32 columns)    x = S scale s_k    p = 2^(x - m)    O^T += C_v^T (P s_v)
// A code has at most eight significant bits, so it is a bfloat16 exactly, and the products run on the matrix cores' bfloat16 form for every type
// of q: q is cut into one (bfloat16), two (binary16) or three (fp32) bfloat16 parts whose products are added, exactly, probabilities into two parts, to
// 2^-16 of themselves, for fp32 three, exactly.
// Bound: long caches by reading the codes once, a few dozen queries each by the vector unit's work on scores and codes (360 instructions a tile of
// 64 binary16 elements beside 16 matrix products), short caches by a wavefront's trips to memory.  Measured: one query to each of 24 caches of 2000 to
// 65536 keys, 16 heads over 2 of 128, bfloat16 over e4m3, 0.41 GB: 92 us and 6.7 for the join, 4.5 TB/s in the former; 61 queries to each of 48 of 100 to
// 4000, 8 heads of 64, binary16 over i8: 62 and 14; one to each of 32 of 12 on average, 4 heads of 32 fp32 with a bias: 10.6.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "tbe_cache.h"

namespace tbe {

// Rows of codes in LDS: chunk c (sixteen bytes) of row r at place (slot(r), c ^ swizzle(r)).  Of 16-byte reads along the rows, those of 16 rows
// fall on 16 different chunks of the 64 banks; of 8-byte reads down the rows (a column of eight rows for each of sixteen lanes), those
// of rows {0 .. 3, 8 .. 11} + 4 (lane / 32) by two chunks.
template <int D>
struct CodeTile {
    static constexpr int kChunks = D / 16;   // of a row: 2, 4 or 8
    static __device__ __forceinline__ int slot(const int r) {   // (an involution)
        return kChunks == 2 ? (r & ~12) | (r & 4) << 1 | (r & 8) >> 1 : r;
    }
    static __device__ __forceinline__ int swizzle(const int s) {   // of the row's slot
        return kChunks == 8 ? ((s >> 3) & 1) << 2 | ((s >> 1) & 1) << 1 | ((s >> 2) & 1) : (kChunks == 4 ? (s >> 2) & 3 : (s >> 3) & 1);
    }
    static __device__ __forceinline__ int place(const int r, const int c) {
        const int s = slot(r);
        return (s * kChunks + (c ^ swizzle(s))) * 16;
    }
    // sixteen codes of row r, chunk c
    static __device__ __forceinline__ uint4 along(const char* lds, const int r, const int c) { return *reinterpret_cast<const uint4*>(lds + place(r, c)); }
    // column 32 t + l % 32 of the eight rows that the registers of fragment m stand for
    static __device__ __forceinline__ uint2 down(const char* lds, const int first, const int m, const int t, const int l) {
        typedef int i32x2_t __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) i32x2_t* lds_ptr;
        const int j = l & 15, r = first + 16 * m + 4 * (l >> 5) + ((j >> 1) & 3) + 8 * (j >> 3), c = 2 * t + ((l >> 4) & 1);
        return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr)(lds + place(r, c) + (j & 1) * 8)));
    }
    // ROWS rows from row j0 of a sequence on, of which there are `rows`, zeros for others, by one wavefront; complete after loads_done()
    template <int ROWS>
    static __device__ __forceinline__ void fetch(char* lds, const char* base, const int64_t stride, const int j0, const int rows, const int dim, const int l) {
        constexpr int kLoads = ROWS * kChunks / 64;
        static_assert(kLoads * 64 == ROWS * kChunks, "whole loads");
        const char* const from = base + (int64_t)j0 * stride;
        const bool whole = j0 + ROWS <= rows && dim == D;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int n = i * 64 + l, s = n / kChunks, r = slot(s), c = (n % kChunks) ^ swizzle(s);
            const char* const src = from + (uint32_t)(r * (uint32_t)stride + c * 16);
            if (whole) load_lds<16>(src, lds + i * 1024);
            else load_lds<16>(j0 + r < rows && c * 16 < dim ? src : reinterpret_cast<const char*>(&attn_zeros), lds + i * 1024);
        }
    }
};

// Eight codes as bfloat16.
template <bool I8>
__device__ __forceinline__ uint4 codes_bf16(const uint32_t lo, const uint32_t hi) {
    if constexpr (I8) {
        float x[8];
        unpack_codes<true>(lo, x);
        unpack_codes<true>(hi, x + 4);
        const bf16_t* const t = nullptr;
        return make_uint4(pack2(t, x[0], x[1]), pack2(t, x[2], x[3]), pack2(t, x[4], x[5]), pack2(t, x[6], x[7]));
    } else {
        return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)));
    }
}

// All bits where the k-th of four e4m3 codes is not a number, none otherwise.
__device__ __forceinline__ uint32_t odd_code(const uint32_t four, const int k) { return 0u - (((four >> (8 * k) & 0x7Fu) + 1u) >> 7); }

// Waits until at most N of this wavefront's loads are under way (vmcnt N, the other counters as they are; see loads_done).
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// How many bfloat16 parts a factor of the type of q has: its significant bits, eight at a time.
template <typename T>
constexpr int parts() { return sizeof(T) == 4 ? 3 : (__is_same(T, bf16_t) ? 1 : 2); }

// ... and a probability times its value's scale: sixteen bits even for bfloat16 results, of whose error a probability rounded to eight would make as much
// as the result's own rounding does (2.4e-3 of the values in the root mean square where this has 1.7e-3).
template <typename T>
constexpr int weight_parts() { return sizeof(T) == 4 ? 3 : 2; }

// Eight factors in parts: each part takes the upper eight bits of what is left, as they are; the last one is rounded.
template <int P>
__device__ __forceinline__ void cut(float (&x)[8], uint4 (&to)[P]) {
    const bf16_t* const t = nullptr;
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if (p == P - 1) {
            to[p] = make_uint4(pack2(t, x[0], x[1]), pack2(t, x[2], x[3]), pack2(t, x[4], x[5]), pack2(t, x[6], x[7]));
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = __float_as_uint(x[2 * i]) & 0xFFFF0000u, b = __float_as_uint(x[2 * i + 1]) & 0xFFFF0000u;
                w[i] = a >> 16 | b;
                x[2 * i] -= __uint_as_float(a);
                x[2 * i + 1] -= __uint_as_float(b);
            }
            to[p] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

struct CacheAttnArgs : AttnArgs {
    const float *ks, *vs;   // [kv][k_rows]
    // The tiles of keys of all sequences, one after the other (a sequence without keys has one too), are shared out in `ranges` runs as long as each
    // other, over the ends of sequences, a run for a wavefront.  qblocks: units of queries of one sequence that go with each run.
    int ranges, qblocks;
    int own;                // a wavefront has a unit of queries and all its keys instead; 2: all queries of a sequence
    int2* spans;            // [N]: the first and the last run of a sequence's keys, the same where there is nothing to join
};

constexpr int kCacheWaves = 4, kCacheThreads = 64 * kCacheWaves;
constexpr int kTileLog2 = 5;   // keys of a tile (heads of 32, 2000 caches of 60 on average: 64 keys 42 us, 32 keys 34; heads of 64: 84 / 82)

// Run r of `ranges` over all `tiles` begins here; the run that a tile belongs to.
__device__ __forceinline__ int64_t range_begin(const int64_t tiles, const int ranges, const int r) { return tiles * r / ranges; }
__device__ __forceinline__ int range_of(const int64_t tiles, const int ranges, const int64_t at) { return (int)(((at + 1) * ranges - 1) / tiles); }

// Where run r begins: the sequence, the number of its first tile, and how many tiles there are in all.  r: of the workgroup's first wavefront, the
// others have the next ones.  All of the workgroup together; every sequence is judged on the way.  An ill-formed sequence counts as one without keys.
struct RangeStart {
    int64_t tiles, begin;
    int s, ranges;   // ranges: as many as there are indeed, since caches may be filled to a small part: none without a tile
};
constexpr int kRangeTiles = 2;   // a run has so many tiles at least
__device__ __forceinline__ int64_t sequence_tiles(const AttnArgs& a, const int s, const int log2) {
    const LaneSequence n = lane_numbers(a, s);
    const int64_t room = n.k1 - n.k0, keys = a.k_len.p ? a.k_len[s] : room;
    if (n.fits && (keys < 0 || keys > room)) *a.err = 1;
    const bool good = n.fits && keys > 0 && keys <= room;
    return good ? (keys + ((int64_t)1 << log2) - 1) >> log2 : 1;
}
__device__ __forceinline__ RangeStart range_start(const CacheAttnArgs& a, const int r, const int log2) {
    __shared__ int64_t waves[kCacheWaves], found_begin[kCacheWaves];
    __shared__ int found[kCacheWaves];
    const int each = (a.N + kCacheThreads - 1) / kCacheThreads, lane = lane_id(), wave = uniform(threadIdx.x >> 6);
    const int s0 = (int)threadIdx.x * each, s1 = s0 + each < a.N ? s0 + each : a.N;
    int64_t mine = 0;
    for (int s = s0; s < s1; ++s) mine += sequence_tiles(a, s, log2);
    int64_t upto = mine;   // ... and of all threads before
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int64_t x = __shfl_up(upto, k);
        if (lane >= k) upto += x;
    }
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    RangeStart out;
    out.tiles = 0;
#pragma unroll
    for (int k = 0; k < kCacheWaves; ++k) {
        if (k < wave) upto += waves[k];
        out.tiles += waves[k];
    }
    const int64_t most = out.tiles / kRangeTiles;
    out.ranges = most < 1 ? 1 : (most < a.ranges ? (int)most : a.ranges);
    for (int k = 0; k < kCacheWaves; ++k) {
        const int64_t at = range_begin(out.tiles, out.ranges, r + k);
        int64_t begin = upto - mine;
        if (at >= begin && at < upto) {
            int s = s0;
            for (; s + 1 < s1; ++s) {
                const int64_t n = sequence_tiles(a, s, log2);
                if (at < begin + n) break;
                begin += n;
            }
            found[k] = s;
            found_begin[k] = begin;
        }
    }
    __syncthreads();
    out.s = uniform(found[wave]);
    out.begin = lane_i64(found_begin[wave], 0);
    out.tiles = lane_i64(out.tiles, 0);
    out.ranges = uniform(out.ranges);
    return out;
}

// What a wavefront does with the part of a sequence's keys that lies in its run.
struct PartWork {
    int block, step, blocks;   // units of queries: the first, how far to the next, the end
    int lo, hi;                // keys
    int cell;                  // 0, 1: where the results go to be joined; -1: these are all keys
};

// Wavefronts of a SIMD that the registers are to leave room for (and the LDS does): heads of 32 2 / 3 / 4, us, 24 caches of 34,000 on average, 16 heads over 2,
// bfloat16 49 / 46 / 47, fp32 53 / 51 / 57;  of 64 2 / 3 62 / 63, 72 / 81 (registers in scratch memory).
constexpr int cache_occupancy(const int D) { return D == 32 ? 3 : 2; }

template <typename T, int D, bool I8, bool BIAS>
__global__ __launch_bounds__(64 * kCacheWaves, cache_occupancy(D)) void cache_attn_kernel(const CacheAttnArgs a) {
    constexpr int kWaves = kCacheWaves, kLog = kTileLog2, BK = 1 << kLog, kT = BK / 32, kD = D / 32, kC = D / 16, kP = parts<T>(), kW = weight_parts<T>();
    constexpr int kTile = BK * D;
    typedef Mma<bf16_t> M;
    typedef CodeTile<D> Codes;
    // two buffers each, as arrays of their own: loads into one of them are seen not to concern what is read from another
    __shared__ __align__(16) char keys0[kWaves * kTile], keys1[kWaves * kTile], values0[kWaves * kTile], values1[kWaves * kTile];
    __shared__ __align__(16) float key_scales0[kWaves * 64], key_scales1[kWaves * 64], value_scales0[kWaves * 64], value_scales1[kWaves * 64];
    extern __shared__ float tab[];
    const int wave = uniform(threadIdx.x >> 6), packs = a.H / a.pack;

    // the heads; the run of keys and the unit of queries that goes with it, or this wavefront's unit of queries
    int hh, qb = 0, r = 0;
    uint32_t v = 0;
    if (a.own) {
        const uint32_t groups = ((uint32_t)a.V + kWaves - 1) / kWaves * (uint32_t)packs, wg = die_order(groups);
        if (wg >= groups) return;
        hh = uniform((int)(wg % (uint32_t)packs));
        v = uniform((int)(wg / (uint32_t)packs * kWaves + wave));
    } else {
        // Runs are dealt to the 8 dies four by four, and each die has all heads and units of queries of its runs, which read the same lines.
        const uint32_t wg = blockIdx.y * gridDim.x + blockIdx.x, each = (uint32_t)packs * a.qblocks, dies = a.ranges >= 8 * kWaves ? 8 : 1;
        const uint32_t n = wg / dies, turn = n / each, rest = n - turn * each;
        r = uniform((int)(turn * dies + wg % dies) * kWaves);
        hh = uniform((int)(rest % (uint32_t)packs));
        qb = uniform((int)(rest / (uint32_t)packs));
        if (r >= a.ranges) return;
    }
    const int head0 = hh * a.pack;
    const bool looks = a.own && v < (uint32_t)a.N && (hh == 0 || a.own == 2);
    const int64_t peek = looks ? sequence_numbers(a, v) : 0;
    if (BIAS) {
        fill_bias(tab, a, head0, a.pack, kCacheThreads);
        __syncthreads();
    }
    int64_t at = 0, end = 1, begin = 0, all = 0;   // own: one turn of the loop below
    int s = 0, ranges = 1;
    if (a.own) {
        if (v >= (uint32_t)a.V) return;
        s = a.own == 2 ? (int)v : find_sequence(a.q_off, a.N, v, a.block);
    } else {
        const RangeStart start = range_start(a, r, kLog);
        s = start.s;
        begin = start.begin;
        all = start.tiles;
        ranges = start.ranges;
        r += wave;
        if (r >= ranges) return;
        at = range_begin(all, ranges, r);
        end = range_begin(all, ranges, r + 1);
    }
    int64_t numbers = a.own == 2 ? peek : (at < end ? sequence_numbers(a, s) : 0);
    for (; at < end; ++s) {
    Sequence q;
    PartWork w;
    const bool fits = take_sequence(a, s, numbers, q);
    if (!a.own) numbers = s + 1 < a.N ? sequence_numbers(a, s + 1) : 0;   // (under way while this one is worked on)
    if (a.own == 2) {
        if (!fits) return;
        w.block = 0;
        w.blocks = (int)(((int64_t)q.nq + a.block - 1) / a.block);
        w.step = 1;
        w.lo = 0;
        w.hi = q.nk;
        w.cell = -1;
        at = end;
    } else if (a.own) {
        const uint32_t start = (uint32_t)q.q0 / a.block + s, blocks = ((uint32_t)q.nq + a.block - 1) / a.block;
        if (!fits || v < start || v - start >= blocks) return judge(a, looks, v, peek);
        w.block = uniform((int)(v - start));
        w.blocks = w.block + 1;
        w.step = 1;
        w.lo = 0;
        w.hi = q.nk;
        w.cell = -1;
        at = end;
    } else {
        const int64_t n = fits && q.nk > 0 ? ((int64_t)q.nk + BK - 1) >> kLog : 1;
        const int64_t a0 = at - begin, a1 = end - begin < n ? end - begin : n;   // tiles of this sequence
        w.blocks = (int)(((int64_t)q.nq + a.block - 1) / a.block);
        w.block = qb;
        w.step = a.qblocks;
        w.lo = (int)(a0 << kLog);
        w.hi = a1 < n ? (int)(a1 << kLog) : q.nk;
        w.cell = a0 > 0 ? 0 : (a1 < n ? 1 : -1);
        if (w.blocks > a.qblocks) {
            // More units of queries than go with a run: units in turn, with all the keys.  Turn m belongs to the run with tile m n / turns.
            const int64_t turns = (w.blocks + a.qblocks - 1) / a.qblocks, m0 = (a0 * turns + n - 1) / n, m1 = (a1 * turns + n - 1) / n;
            w.block = (int)m0 * a.qblocks + qb;
            w.blocks = w.blocks < (int)m1 * a.qblocks ? w.blocks : (int)m1 * a.qblocks;
            w.lo = 0;
            w.hi = q.nk;
            w.cell = -1;
        }
        if (a0 == 0 && hh == 0 && qb == 0 && lane_id() == 0)
            a.spans[s] = w.cell < 0 ? make_int2(0, 0) : make_int2(r, range_of(all, ranges, begin + n - 1));
        begin += n;
        at = begin;
        if (!fits) continue;
    }

    const int kvh = head0 / a.group;
    const char* const kb = a.k.at(q.k0, kvh);
    const char* const vb = a.v.at(q.k0, kvh);
    const float* const ks = a.ks + (int64_t)kvh * a.k_rows + q.k0;
    const float* const vs = a.vs + (int64_t)kvh * a.k_rows + q.k0;
    const int own = wave * kTile, own_scales = wave * 64;
    for (int block = w.block; block < w.blocks; block += w.step) {
        const int lane = anew(lane_id()), col = lane & 31, half = lane >> 5;
        const int ci = col / a.pack, cg = col - ci * a.pack, head = head0 + cg;
        const int iw = block * a.block, i = iw + ci;
        float beyond = 0.f, ahead = 0.f;
        const float* const ht = tab + cg * tab_size(a.far);
        if (BIAS) {
            beyond = ht[kTabMargin];
            ahead = a.causal ? 0.f : ht[2 * a.far + kTabMargin];
        }
        const bool is = ci < a.qpt && i < q.nq;
        const int first = q.nk - q.nq + iw, pos = first + ci, wave_last = first + a.qpt - 1;   // places among the keys
        int jend = w.hi;   // keys of this unit: all that its last query sees
        if (a.causal) {
            const int last = q.nk - q.nq + (iw + a.block < q.nq ? iw + a.block : q.nq);
            jend = jend < last ? jend : last;
        }
        const int tiles = jend > w.lo ? (jend - w.lo + BK - 1) / BK : 0;

        uint4 fq[kC][kP];   // fragment 2 c + s: elements 32 c + 16 half + 8 s + 0 .. 7, the order in which a chunk of codes has them
        {
            const char* const row = a.q.at(q.q0 + (is ? i : 0), head);
#pragma unroll
            for (int n = 0; n < kC; ++n) {
                const int e = 32 * (n / 2) + 16 * half + 8 * (n % 2);
                const bool there = is && e < a.dim;
                float x[8];
                if constexpr (sizeof(T) == 4) {
                    const float4 u = *reinterpret_cast<const float4*>(row + (there ? e : 0) * 4), y = *reinterpret_cast<const float4*>(row + (there ? e + 4 : 0) * 4);
                    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
                    x[4] = y.x; x[5] = y.y; x[6] = y.z; x[7] = y.w;
                } else {
                    Frag<T>::unpack(*reinterpret_cast<const uint4*>(row + (there ? e : 0) * 2), x);
                }
                uint4 odd;   // what is not finite is its own first part, and has no other
                float f[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    x[k] = there ? (a.negative ? -x[k] : x[k]) : 0.f;
                    const bool finite = fabsf(x[k]) < __builtin_inff();
                    f[k] = finite ? 0.f : x[k];
                    x[k] = finite || kP == 1 ? x[k] : 0.f;
                }
                const bf16_t* const t = nullptr;
                odd = make_uint4(pack2(t, f[0], f[1]), pack2(t, f[2], f[3]), pack2(t, f[4], f[5]), pack2(t, f[6], f[7]));
                cut<kP>(x, fq[n]);
                if constexpr (kP > 1) {
                    fq[n][0].x |= odd.x; fq[n][0].y |= odd.y; fq[n][0].z |= odd.z; fq[n][0].w |= odd.w;
                }
            }
        }

        f32x16_t o[kD];
        float m, sum, lift = 0.f;   // lift: see below
        auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int d = 0; d < kD; ++d) o[d] = f32x16_t{};
            m = -__builtin_inff();
            sum = 0.f;
        };
        auto fetch = [&](const int t, char* const to, float* const st, const char* const from, const int64_t stride, const float* const scales, const int l) __attribute__((always_inline)) {
            const int j0 = w.lo + t * BK, j = j0 + (l & (BK - 1));
            Codes::template fetch<BK>(to + own, from, stride, j0, q.nk, a.dim, l);
            load_lds<4>(j < q.nk ? reinterpret_cast<const char*>(scales + j) : reinterpret_cast<const char*>(&attn_zeros), st + own_scales);
        };
        auto fetch_keys = [&](const int t, char* const to, float* const st, const int l) __attribute__((always_inline)) { fetch(t, to, st, kb, a.k.row, ks, l); };
        auto fetch_values = [&](const int t, char* const to, float* const st, const int l) __attribute__((always_inline)) { fetch(t, to, st, vb, a.v.row, vs, l); };
        f32x16_t x[kT];   // a tile's scores
        auto scores = [&](const int t, const char* const kt_, const float* const st_, const int l) __attribute__((always_inline)) {
            const int j0 = w.lo + t * BK, col = l & 31, half = l >> 5;
            const char* const kt = kt_ + own;
            const float* const st = st_ + own_scales;
#pragma unroll
            for (int k = 0; k < kT; ++k) {
                x[k] = f32x16_t{};
#pragma unroll
                for (int c = 0; c < kC / 2; ++c) {
                    const uint4 u = Codes::along(kt, 32 * k + col, 2 * c + half);
                    const uint4 f0 = codes_bf16<I8>(u.x, u.y), f1 = codes_bf16<I8>(u.z, u.w);
#pragma unroll
                    for (int p = kP - 1; p >= 0; --p) {
                        x[k] = M::mma(f0, fq[2 * c][p], x[k]);
                        x[k] = M::mma(f1, fq[2 * c + 1][p], x[k]);
                    }
                }
            }
            settle<bf16_t>();
            const bool hides = j0 + BK > q.nk || (a.causal && j0 + BK - 1 > first);
#pragma unroll
            for (int k = 0; k < kT; ++k) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 s = *reinterpret_cast<const float4*>(st + 32 * k + 2 * r + 4 * half);
                    x[k][r] *= s.x; x[k][r + 1] *= s.y; x[k][r + 2] *= s.z; x[k][r + 3] *= s.w;
                }
                if (BIAS) {
                    // A bias of -infinity hides a score that is not finite too.  (The sum as a value that the compiler has to have before it selects: it made
                    // a branch between the lanes of one of sixteen; see column_row.)
                    const auto add = [&](float& y, const float b) __attribute__((always_inline)) {
                        float z = fmaf(y, a.scale2, b);
                        asm volatile("" : "+v"(z));
                        y = b == -__builtin_inff() ? b : z;
                    };
                    const int j = j0 + 32 * k;
                    if (first - (j + 31) >= a.far || wave_last - j <= -a.far) {
                        const float b = first - (j + 31) >= a.far ? beyond : ahead;
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            float y = x[k][r];
                            add(y, b);
                            x[k][r] = y;
                        }
                    } else {
                        const float* const from = ht + (j + 4 * half - pos + a.far + kTabMargin);
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            float y = x[k][r];
                            add(y, from[8 * (r / 4) + r % 4]);
                            x[k][r] = y;
                        }
                    }
                }
            }
            if (hides) {
                const int upto = a.causal && pos + 1 < q.nk ? pos + 1 : q.nk;   // the keys that this column sees end here
#pragma unroll
                for (int k = 0; k < kT; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        float y = x[k][r];
                        asm volatile("" : "+v"(y));   // (no branch, as above)
                        x[k][r] = j0 + 32 * k + 8 * (r / 4) + 4 * half + r % 4 >= upto ? -__builtin_inff() : y;
                    }
            }
            return hides;
        };
        auto apply = [&](const char* const vt_, const float* const st_, const bool hides, const int l, const auto lifted) __attribute__((always_inline)) {
            const int half = l >> 5;
            const char* const vt = vt_ + own;
            const float* const st = st_ + own_scales;
            float top = -__builtin_inff();
#pragma unroll
            for (int k = 0; k < kT; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, x[k][r]);
            top = halves_max(top);
            if (!BIAS) top *= a.scale2;
            // A maximum that grows by less than 2^8 is left as it is: the probabilities stay below 2^8, and what they are divided by in the end is
            // added up from them.
            if (__any(top > m + 8.f)) {
                const float grown = fmaxf(m, top);
                const float shrink = grown == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(m - grown);
                m = grown;
                sum *= shrink;
#pragma unroll
                for (int d = 0; d < kD; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
            }
            float at = m == -__builtin_inff() ? 0.f : m;   // (nothing seen so far: every probability is 2^-inf = 0)
            if constexpr (decltype(lifted)::value) at += lift;
            // A scale that is not finite must not reach a column that does not see its key.
            const auto weigh = [&](const auto masked) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < kT; ++k)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const float4 s4 = *reinterpret_cast<const float4*>(st + 32 * k + 2 * r + 4 * half);
                        const float s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float y = x[k][r + e], p = __builtin_amdgcn_exp2f(BIAS ? y - at : fmaf(y, a.scale2, -at));
                            sum += p;
                            x[k][r + e] = p * (decltype(masked)::value && y == -__builtin_inff() ? 0.f : s[e]);
                        }
                    }
            };
            if (BIAS || hides) weigh(std::true_type{});
            else weigh(std::false_type{});
#pragma unroll
            for (int k = 0; k < kT; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float p[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) p[r] = x[k][8 * c + r];
                    uint4 f[kW];
                    cut<kW>(p, f);
#pragma unroll
                    for (int d = 0; d < kD; ++d) {
                        const uint2 u = Codes::down(vt, 32 * k, c, d, l);
                        const uint4 g = codes_bf16<I8>(u.x, u.y);
#pragma unroll
                        for (int n = kW - 1; n >= 0; --n) o[d] = M::mma(g, f[n], o[d]);
                    }
                }
            settle<bf16_t>();
        };
        // Codes that are not numbers (e4m3) among the values: a column that does not see their key would get 0 times them from the matrix cores.  They
        // are taken out of the tile, and the columns that see the key get NaN where they stood.
        auto take_out = [&](const int t, const int l) __attribute__((always_inline)) {
            const int j0 = w.lo + t * BK, half = l >> 5;
            char* const vt = values0 + own;
            const int upto = a.causal && pos + 1 < q.nk ? pos + 1 : q.nk;
#pragma unroll 1
            for (int j = 0; j < BK; ++j) {
                const int key = j0 + j;
                bool sees = key < upto;
                if (BIAS) {
                    int d = pos - key;
                    d = d > a.far ? a.far : (d < -a.far ? -a.far : d);
                    sees = sees && ht[a.far + kTabMargin - d] != -__builtin_inff();
                }
                const uint32_t seen = sees ? ~0u : 0u;
#pragma unroll
                for (int d = 0; d < kD; ++d)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const int e = 32 * d + 8 * n + 4 * half;
                        const uint32_t u = *reinterpret_cast<const uint32_t*>(vt + Codes::place(j, e / 16) + e % 16);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t b = u >> (8 * k) & 0x7Fu & seen;
                            asm volatile("" : "+v"(b));   // (no branch, as above)
                            o[d][4 * n + k] = b == 0x7Fu ? __builtin_nanf("") : o[d][4 * n + k];
                        }
                    }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
            for (int n = l; n < kTile / 4; n += 64) {
                uint32_t u = *reinterpret_cast<const uint32_t*>(vt + 4 * n);
#pragma unroll
                for (int k = 0; k < 4; ++k) u &= ~(odd_code(u, k) & 0xFFu << (8 * k));
                *reinterpret_cast<uint32_t*>(vt + 4 * n) = u;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        };

        // Two tiles of keys and of values are under way or in use; a buffer is filled anew as soon as its tile has been multiplied, so that the loads have
        // a tile's time and a half (24 caches of long histories: 120 us where the next tile is asked for when this one is there, 93 so; 82 for the loads alone).
        // They end in their order: of those begun after the ones waited for, so many may still run.
        constexpr int kGroup = BK * D / 1024 + 1;
        auto one = [&](const int t, char* const kt, float* const kst, char* const vt, float* const vst) __attribute__((always_inline)) {
            const bool next = t + 1 < tiles, after = t + 2 < tiles;
            if (next) wait_loads<3 * kGroup>();
            else wait_loads<kGroup>();
            const bool hides = scores(t, kt, kst, lane);
            if (after) {
                fetch_keys(t + 2, kt, kst, lane);
                wait_loads<3 * kGroup>();
            } else if (next) {
                wait_loads<2 * kGroup>();
            } else {
                wait_loads<0>();
            }
            apply(vt, vst, hides, lane, std::false_type{});
            if (after) fetch_values(t + 2, vt, vst, lane);
        };
        begin();
        if (tiles > 0) {
            fetch_keys(0, keys0, key_scales0, lane);
            fetch_values(0, values0, value_scales0, lane);
        }
        if (tiles > 1) {
            fetch_keys(1, keys1, key_scales1, lane);
            fetch_values(1, values1, value_scales1, lane);
        }
        for (int t = 0; t < tiles; t += 2) {
            one(t, keys0, key_scales0, values0, value_scales0);
            if (t + 1 < tiles) one(t + 1, keys1, key_scales1, values1, value_scales1);
        }
        if (__any(is && not_finite(o))) {
            // Codes that are not numbers, see above; or, since a probability counts up to 2^8 until it is divided by the sum of all, sums of values near fp32's
            // largest beyond it.  The columns that are not finite then get a maximum that is greater by `lift`, whose probabilities are that much smaller: no more than
            // the largest scale here and the number of keys ask for, as small values beside those lose their last bits to it.
            const int odd = not_finite(o);
            float top = 0.f;
#pragma unroll 1
            for (int j = w.lo; j < jend; j += 64) {
                const int n = j + lane < jend ? j + lane : jend - 1;
                const float x = fabsf(vs[n]);
                top = x < __builtin_inff() ? fmaxf(top, x) : top;
            }
            const int e = wave_max_i32((int)(__float_as_uint(top) >> 23)) - 126;   // scales are below 2^e, codes below 2^9
            const int over = uniform(e + 9 + 8 + (32 - __builtin_clz(jend - w.lo)) + 1 - 128);
            lift = (odd | __shfl_xor(odd, 32)) && over > 0 ? (float)over : 0.f;
            if (over > 0 || (!I8 && (a.causal || BIAS))) {
                begin();
#pragma unroll 1
                for (int t = 0; t < tiles; ++t) {
                    const int l = anew(lane);   // (few registers: nothing of this is kept through the loop above)
                    fetch_keys(t, keys0, key_scales0, l);
                    fetch_values(t, values0, value_scales0, l);
                    loads_done();
                    if (!I8 && (a.causal || BIAS)) take_out(t, l);
                    const bool hides = scores(t, keys0, key_scales0, l);
                    apply(values0, value_scales0, hides, l, std::true_type{});
                }
                m += lift;
            }
        }
        sum = pair_sum<32>(sum);

        if (!is) continue;
        if (w.cell >= 0) {
            const int64_t cell = (((int64_t)(2 * r + w.cell) * a.qblocks + qb) * packs + hh) * 32 + col;
            if (half == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * cell) = make_float2(m, sum);
            float* const to = a.part_o + cell * D + 4 * half;
#pragma unroll
            for (int d = 0; d < kD; ++d)
#pragma unroll
                for (int n = 0; n < 16; n += 4) *reinterpret_cast<float4*>(to + 32 * d + 2 * n) = make_float4(o[d][n], o[d][n + 1], o[d][n + 2], o[d][n + 3]);
            continue;
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (no key seen: zeros)
        char* const to = const_cast<char*>(a.o.at(q.q0 + i, head));
#pragma unroll
        for (int d = 0; d < kD; ++d)
#pragma unroll
            for (int n = 0; n < 16; n += 4) {
                const int e = 32 * d + 2 * n + 4 * half;
                if (e < a.dim) {
                    if constexpr (sizeof(T) == 2)
                        *reinterpret_cast<uint2*>(to + 2 * e) = make_uint2(pack2((const T*)nullptr, o[d][n] * inv, o[d][n + 1] * inv),
                                                                           pack2((const T*)nullptr, o[d][n + 2] * inv, o[d][n + 3] * inv));
                    else *reinterpret_cast<float4*>(to + 4 * e) = make_float4(o[d][n] * inv, o[d][n + 1] * inv, o[d][n + 2] * inv, o[d][n + 3] * inv);
                }
            }
        if (a.lse && half == 0) a.lse[(int64_t)head * a.q_rows + q.q0 + i] = sum == 0.f ? -__builtin_inff() : fmaf(m, kLn2, logf(sum));
    }
    }
    if (a.own == 1) judge(a, looks, v, peek);
}

// Joins the parts of the keys: a workgroup for eight heads of a query, a wavefront for two of them, or where there are many parts for one head.  A row
// of a part is shared by D / 4 lanes, and the lanes' groups take parts in turn, each with its own running maximum: the rows are loaded beside the
// statistics that weigh them.  The order of the additions is fixed.
template <typename T, int D, bool many>
__global__ __launch_bounds__(256, many ? 4 : 8) void cache_attn_join_kernel(const CacheAttnArgs a) {
    constexpr int kLanes = D / 4, kGroups = 64 / kLanes, kAhead = many ? 8 : 4;   // kAhead: parts of a group under way together
    __shared__ float2 stats[4];
    __shared__ float4 sums[4][kLanes];
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), packs = a.H / a.pack;
    const int heads = many ? 1 : 8;
    const uint32_t n = blockIdx.y * gridDim.x + blockIdx.x, per_row = ((uint32_t)a.H + heads - 1) / heads;
    const int64_t row = n / per_row;
    const int head0 = (int)(n - (uint32_t)row * per_row) * heads;
    if (row >= a.q_rows) return;
    const int s = find_row(a.q_off, a.N, row);
    Sequence q;
    const int2 span = a.spans[s];
    if (!take_sequence(a, s, sequence_numbers(a, s), q) || row < q.q0 || row >= q.q0 + q.nq) return;
    if (span.x >= span.y) return;   // (the result is there already)
    const int i = (int)(row - q.q0), qb = i / a.block, count = span.y - span.x + 1;
    const int64_t each = (int64_t)a.qblocks * packs * 32;   // cells of half a run's: a run has two, for the sequence that it continues and the one that it begins
    const int e0 = 4 * (lane % kLanes), group = lane / kLanes + (many ? wave * kGroups : 0), groups = many ? 4 * kGroups : kGroups;
    for (int head = head0 + (many ? 0 : wave); head < a.H && head < head0 + heads; head += 4) {
        const int hh = head / a.pack, col = (i - qb * a.block) * a.pack + head - hh * a.pack;
        const int64_t cell0 = ((int64_t)qb * packs + hh) * 32 + col;
        float m, sum;
        float4 o;
        const auto add = [&](const float2 c, const float4 x) __attribute__((always_inline)) {
            const float top = fmaxf(m, c.x), at = top == -__builtin_inff() ? 0.f : top;
            const float old = __builtin_amdgcn_exp2f(m - at), by = __builtin_amdgcn_exp2f(c.x - at);
            m = top;
            sum = fmaf(c.y, by, sum * old);
            o.x = fmaf(x.x, by, o.x * old); o.y = fmaf(x.y, by, o.y * old);
            o.z = fmaf(x.z, by, o.z * old); o.w = fmaf(x.w, by, o.w * old);
        };
        const auto join = [&](const auto small) __attribute__((always_inline)) {   // small: of the parts' results times 2^-12
            m = -__builtin_inff();
            sum = 0.f;
            o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int base = group; base < count; base += groups * kAhead) {
                float2 c[kAhead];
                float4 x[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    const int p = base + j * groups < count ? base + j * groups : base;
                    const int64_t cell = cell0 + (2 * (int64_t)(span.x + p) + (p == 0)) * each;
                    c[j] = *reinterpret_cast<const float2*>(a.part_ml + 2 * cell);
                    x[j] = *reinterpret_cast<const float4*>(a.part_o + cell * D + e0);
                }
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    if constexpr (decltype(small)::value) x[j] = make_float4(x[j].x * 0x1p-12f, x[j].y * 0x1p-12f, x[j].z * 0x1p-12f, x[j].w * 0x1p-12f);
                    if (base + j * groups < count) add(c[j], x[j]);
                }
            }
#pragma unroll
            for (int w = kLanes; w < 64; w <<= 1) {
                const float2 c = make_float2(__shfl_xor(m, w), __shfl_xor(sum, w));
                const float4 x = make_float4(__shfl_xor(o.x, w), __shfl_xor(o.y, w), __shfl_xor(o.z, w), __shfl_xor(o.w, w));
                add(c, x);
            }
            if (many) {
                if (lane == 0) stats[wave] = make_float2(m, sum);
                if (lane < kLanes) sums[wave][lane] = o;
                __syncthreads();
                m = -__builtin_inff();
                sum = 0.f;
                o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < 4; ++w) add(stats[w], sums[w][lane % kLanes]);
            }
        };
        join(std::false_type{});
        // Parts of values near fp32's largest may add up beyond it before they are divided by their weights: fewer than 2^12 parts.  (In a workgroup that has one
        // head together, all wavefronts find the same here.)
        float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (__any(!(fabsf(o.x) < __builtin_inff() && fabsf(o.y) < __builtin_inff() && fabsf(o.z) < __builtin_inff() && fabsf(o.w) < __builtin_inff()))) {
            const float4 first = o;
            if (many) __syncthreads();
            join(std::true_type{});
            const auto pick = [&](const float x, const float y) { return fabsf(x) < __builtin_inff() ? x * inv : y * inv * 0x1p12f; };
            o = make_float4(pick(first.x, o.x), pick(first.y, o.y), pick(first.z, o.z), pick(first.w, o.w));
            inv = 1.f;
        }
        if (many && wave != 0) return;
        if (lane < kLanes && e0 < a.dim) {
            char* const to = const_cast<char*>(a.o.at(row, head)) + e0 * sizeof(T);
            if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack2((const T*)nullptr, o.x * inv, o.y * inv), pack2((const T*)nullptr, o.z * inv, o.w * inv));
            else *reinterpret_cast<float4*>(to) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        }
        if (a.lse && lane == 0) a.lse[(int64_t)head * a.q_rows + row] = sum == 0.f ? -__builtin_inff() : fmaf(m, kLn2, logf(sum));
    }
}

// How the work is shared out.  Heads of a group lie side by side in a wavefront's columns where one query would leave them empty.  Short caches, or
// middling ones of enough sequences: a wavefront for each unit of queries, with all its keys.  Otherwise as many wavefronts as the chip holds at once
// share all keys evenly, whosesoever they are, and what was cut is joined.  On their own / shared evenly, us, one query to each of so many caches
// of that many keys on average (half to one and a half times as many), 32 heads of 128 over 8, bfloat16 over e4m3:
//   8 of 128 17 / 22, of 256 24 / 22, of 2048 132 / 28;  32 of 256 25 / 25, of 512 40 / 28;  128 of 256 26 / 35, of 512 43 / 52, of 1024 76 / 82, of 2048 142 /
//   140;  512 of 128 48 / 70, of 512 131 / 162;  1024 of 256 130 / 177
// 4 heads of 32: 32 of 512 25 / 23, 256 of 512 27 / 34, of 1024 44 / 42;  61 queries each, 8 heads of 64, binary16 over i8: 8 of 256 23 / 26, 48 of 256 28 / 44, of
// 1024 74 / 61.
// Evenly among 512 workgroups, two wavefronts a SIMD (heads of 32: 768); among 256 where the codes' conversions are the cheapest (e4m3 into bfloat16
// products), heads have 128 elements and runs are long, since memory then bounds it and fewer streams serve it better: 512 / 256, us, 24 caches of
// 34,000 on average, 16 heads over 2 of 128 bfloat16 102 / 100 (two queries each 104 / 101, four 111 / 105, with a bias 128 / 111), 64 of 2250, 32 heads over 8 93 / 89,
// 128 of 2048 142 / 133;  but over i8 105 / 111, binary16 over i8 111 / 119, fp32 134 / 158, heads of 64 68 / 75, 8 of 2048 29 / 33 and 61 queries each to 48 of 1024,
// 8 heads of 64, 54 / 63.
// Many queries are shared out evenly too (on their own / evenly: 1024 to each of 4 of 4500, 16 heads over 4 of 128, 574 / 277 us; 2048 to one of 8000, 32 heads
// over 8, 773 / 536; 2048 to each of 8 of 4000, 16 heads over 4 of 64, 832 / 699), as long as the parts' results take no more than some 0.5 GB.
// What decides is the average, so that one cache that is far longer than the others of a batch of short ones is walked by one wavefront (for every head,
// or heads side by side). On their own / evenly, us, 1000 of 240 of which one has 3000, 10,000, 60,000, 32 heads of 128 over 8: 165 / 173, 477 / 175, 2770 / 207;
// 8 heads of 32 over 4: 87 / 49, 269 / 48, 1577 / 58.
constexpr int64_t kMostEach = 4096;
constexpr int64_t kRangeGroups = 512, kRangeGroupsLight = 256, kLongRun = 16;   // kLongRun: tiles
CacheAttnPlan cache_attn_plan(const AttnShape& sh, const bool light, const int max_pack) {
    CacheAttnPlan p;
    const int64_t mean_q = (sh.q_rows + sh.N - 1) / sh.N, mean_k = (sh.k_rows + sh.N - 1) / sh.N;
    p.D = sh.dim <= 32 ? 32 : (sh.dim <= 64 ? 64 : 128);
    p.pack = 1;
    const int group = sh.H / sh.kv;
    const int64_t table = sh.buckets ? (2 * (int64_t)sh.far + 1 + 2 * kTabMargin) * 4 : 0;
    for (int g = 2; g <= group && g <= max_pack; ++g)   // more heads side by side as long as a sequence's queries of all of them fit
        if (group % g == 0 && mean_q * g <= 32 && g * table <= kTabBytes) p.pack = g;
    p.block = 32 / p.pack;
    const int64_t packs = sh.H / p.pack, units = (sh.q_rows == sh.N ? sh.N : sh.q_rows / p.block + sh.N / 2) * packs;
    p.direct = sh.q_rows == sh.N;
    p.qblocks = (int)std::max<int64_t>(1, (mean_q + p.block - 1) / p.block);
    const int64_t each = packs * p.qblocks;   // workgroups that go with a run
    p.own = mean_k <= 320 || (units >= 768 && mean_k <= (p.direct ? 1024 : 512)) || each > kMostEach;
    p.ranges = 1;
    p.V = p.direct ? sh.N : sh.q_rows / p.block + sh.N;
    p.spans = p.part_ml = p.part_o = 0;
    if (p.own) return p;
    const int64_t tiles = (sh.k_rows >> kTileLog2) + sh.N;
    const bool few = light && p.D == 128 && p.qblocks == 1 && tiles * each >= kLongRun * kRangeGroups * kCacheWaves;
    p.ranges = (int)std::max<int64_t>(1, (few ? kRangeGroupsLight : kRangeGroups * cache_occupancy(p.D) / 2) / each) * kCacheWaves;
    if (p.ranges >= 8 * kCacheWaves) p.ranges &= ~(8 * kCacheWaves - 1);
    // no shorter than a few tiles
    p.ranges = (int)std::max<int64_t>(1, std::min<int64_t>(p.ranges, tiles / kRangeTiles));
    p.spans = ((size_t)sh.N * sizeof(int2) + 255) & ~(size_t)255;
    const int64_t cells = p.ranges > 1 ? 2 * p.ranges * each * 32 : 0;
    p.part_ml = ((size_t)cells * 8 + 255) & ~(size_t)255;
    p.part_o = ((size_t)cells * p.D * 4 + 255) & ~(size_t)255;
    return p;
}
static int64_t plan_groups(const AttnShape& sh, const CacheAttnPlan& p) {
    const int64_t packs = sh.H / p.pack;
    return p.own ? (p.V + 3) / 4 * packs : (p.ranges >= 8 * kCacheWaves ? (p.ranges + 8 * kCacheWaves - 1) / (8 * kCacheWaves) * 8 : ((int64_t)p.ranges + kCacheWaves - 1) / kCacheWaves) * packs * p.qblocks;
}
bool cache_attn_grid_ok(const AttnShape& sh, const CacheAttnPlan& p) {
    const int64_t most = ((int64_t)1 << 31) - 64;
    return plan_groups(sh, p) < most && (p.part_ml == 0 || sh.q_rows * sh.H < most);
}
size_t cache_attn_workspace(const AttnShape& sh) {
    size_t most = 0;
    for (int pack = 1; pack <= 32; ++pack) {   // (how many heads go side by side depends on the bias)
        AttnShape any = sh;
        any.far = 0;
        const CacheAttnPlan p = cache_attn_plan(any, false, pack);
        most = std::max(most, p.spans + p.part_ml + p.part_o);
    }
    return most;
}

template <typename T, int D, bool I8>
static hipError_t launch_parts(const tbe_handle* h, const CacheAttnArgs& a, const uint64_t groups, hipStream_t s) {
    hipError_t e;
    {
        LaunchTimer tm(h, s, "cache_attention");
        if (a.bias) cache_attn_kernel<T, D, I8, true><<<die_grid(groups), 64 * kCacheWaves, (size_t)a.pack * (2 * a.far + 1 + 2 * kTabMargin) * 4, s>>>(a);
        else cache_attn_kernel<T, D, I8, false><<<die_grid(groups), 64 * kCacheWaves, 0, s>>>(a);
        e = hipGetLastError();
        tm.done();
    }
    return e;
}
template <typename T, int D>
static hipError_t launch_dim(const tbe_handle* h, const CacheAttnArgs& a, const bool i8, const uint64_t groups, const int join, hipStream_t s) {
    const hipError_t e = i8 ? launch_parts<T, D, true>(h, a, groups, s) : launch_parts<T, D, false>(h, a, groups, s);
    if (e != hipSuccess || !join) return e;
    LaunchTimer tm(h, s, "cache_attention_join");
    if (join == 2) cache_attn_join_kernel<T, D, true><<<die_grid((uint64_t)a.q_rows * (uint64_t)a.H), 256, 0, s>>>(a);
    else cache_attn_join_kernel<T, D, false><<<die_grid((uint64_t)a.q_rows * (((uint64_t)a.H + 7) / 8)), 256, 0, s>>>(a);
    tm.done();
    return hipGetLastError();
}
template <typename T>
static hipError_t launch_type(const tbe_handle* h, const CacheAttnArgs& a, const int D, const bool i8, const uint64_t groups, const int join, hipStream_t s) {
    return D == 32 ? launch_dim<T, 32>(h, a, i8, groups, join, s) : (D == 64 ? launch_dim<T, 64>(h, a, i8, groups, join, s) : launch_dim<T, 128>(h, a, i8, groups, join, s));
}

hipError_t launch_cache_attention(const tbe_handle* h, const AttnArgs& call, const CodeRows (&cache)[2], const bool i8, const CacheAttnPlan& p, const int io,
                                  void* workspace, hipStream_t s) {
    CacheAttnArgs a{};
    static_cast<AttnArgs&>(a) = call;
    a.k = cache[0].codes; a.v = cache[1].codes;
    a.ks = cache[0].scales; a.vs = cache[1].scales;
    a.pack = p.pack; a.qpt = a.block = p.block; a.V = (int)p.V;
    a.ranges = p.ranges; a.qblocks = p.qblocks; a.own = p.own ? 1 + p.direct : 0;
    a.spans = static_cast<int2*>(workspace);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.spans);
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.spans + p.part_ml);
    AttnShape sh{};
    sh.H = a.H;
    const uint64_t groups = (uint64_t)plan_groups(sh, p);
    // 2: many parts of each sequence, a workgroup for a head (24 long histories in 43 parts each, 8 heads a workgroup / one: 17 / 8 us)
    const int join = p.part_ml > 0 ? (p.ranges > 16 * (int64_t)a.N ? 2 : 1) : 0;
    return io == 0 ? launch_type<float>(h, a, p.D, i8, groups, join, s) : (io == 1 ? launch_type<__half>(h, a, p.D, i8, groups, join, s) : launch_type<bf16_t>(h, a, p.D, i8, groups, join, s));
}

}  // namespace tbe
