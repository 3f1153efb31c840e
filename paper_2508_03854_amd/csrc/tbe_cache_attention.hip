// Attention over a cache of one byte an element (see tbe355.h): the keys' and values' codes are multiplied as they are, their scales where the scores and
// probabilities are in fp32 anyway; no value of the cache is ever written out.
//   S^T = C_k Q^T  (a tile: 32 keys x 32 columns)    x = S scale s_k    p = 2^(x - m)    O^T += C_v^T (P s_v)
// A code has at most eight significant bits, so it is a bfloat16 exactly, and the products run on the matrix cores' bfloat16 form for every type
// of q: a binary16 or fp32 factor is cut into two or three bfloat16 parts whose products are added (q exactly, probabilities to 2^-16 of
// themselves or exactly).  bfloat16 probabilities are rounded once.
// Bound: reading the codes once; 24 caches of long histories are 0.4 GB.
#include <hip/hip_runtime.h>

#include <algorithm>

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

// How many bfloat16 parts a factor of the type of q has: its significant bits, eight at a time.
template <typename T>
constexpr int parts() { return sizeof(T) == 4 ? 3 : (__is_same(T, bf16_t) ? 1 : 2); }

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
    // Parts of the keys: a sequence's rows in the cache are cut every 2^cut_log2 of them; part v of the cache belongs to sequence s if s owns it as it
    // would own a unit of queries (see find_sequence).  qblocks: units of queries of one sequence that are handed out with each part.
    int cut_log2, qblocks;
    int own;                // a wavefront has a unit of queries and all its keys instead
};

// The sequence of part v.  All lanes of a wavefront together, 64 offsets at a time.
__device__ __forceinline__ int find_part(const IdxView off, const int N, const uint32_t v, const int cut_log2) {
    int lo = 0, hi = N;
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, s = lo + lane_id() * step;
        const uint64_t m = __ballot(s < hi && (off[s] >> cut_log2) + s <= (int64_t)v);
        const int k = m ? 63 - __builtin_clzll(m) : 0;
        lo += k * step;
        hi = hi < lo + step ? hi : lo + step;
    }
    return uniform(lo);
}

// What a part of the keys has to do.
struct PartWork {
    int block, step, blocks;   // units of queries: the first, how far to the next, the end
    int lo, hi, parts;         // keys; into how many parts the keys of a query are cut
};
__device__ __forceinline__ int part_count(const CacheAttnArgs& a, const int keys) {
    const int n = (int)(((int64_t)keys + ((int64_t)1 << a.cut_log2) - 1) >> a.cut_log2);
    return n < 1 ? 1 : n;
}
// Part n of a sequence, unit qb of those that go with it; false: nothing.  Sequences with more units of queries than go with a part are not cut: their
// parts take units in turn, with all the keys.
__device__ __forceinline__ bool part_work(const CacheAttnArgs& a, const Sequence& q, const int n, const int qb, PartWork& w) {
    w.blocks = (int)(((int64_t)q.nq + a.block - 1) / a.block);
    w.parts = part_count(a, q.nk);
    if (n >= w.parts) return false;
    if (w.blocks > a.qblocks) {
        w.block = n * a.qblocks + qb;
        w.step = w.parts * a.qblocks;
        w.lo = 0;
        w.hi = q.nk;
        w.parts = 1;
    } else {
        w.block = qb;
        w.step = w.blocks > 0 ? w.blocks : 1;
        w.lo = (int)((int64_t)n << a.cut_log2);
        w.hi = w.parts == 1 ? q.nk : (int)(((int64_t)n + 1) << a.cut_log2 < q.nk ? ((int64_t)n + 1) << a.cut_log2 : q.nk);
    }
    return w.block < w.blocks;
}

constexpr int kCacheWaves = 4;
template <int D>
constexpr int cache_tile_rows() { return D == 128 ? 32 : 64; }

template <typename T, int D, bool I8, bool BIAS>
__global__ __launch_bounds__(64 * kCacheWaves, 2) void cache_attn_kernel(const CacheAttnArgs a) {
    constexpr int kWaves = kCacheWaves, BK = cache_tile_rows<D>(), kT = BK / 32, kD = D / 32, kC = D / 16, kP = parts<T>();
    constexpr int kTile = BK * D, kRow = D / 4;
    typedef Mma<bf16_t> M;
    typedef CodeTile<D> Codes;
    // two buffers each, as arrays of their own: loads into one of them are seen not to concern what is read from another
    __shared__ __align__(16) char keys0[kWaves * kTile], keys1[kWaves * kTile], values0[kWaves * kTile], values1[kWaves * kTile];
    __shared__ __align__(16) float scales0[kWaves * 2 * BK], scales1[kWaves * 2 * BK];   // keys' and values' of each wavefront's tile
    __shared__ float2 stats[kWaves * 32];
    extern __shared__ float tab[];
    static_assert(kWaves * kTile >= 32 * D * 4, "a wavefront's results find room in one of the arrays");
    const int wave = uniform(threadIdx.x >> 6), lane = lane_id(), col = lane & 31, half = lane >> 5;
    const int packs = a.H / a.pack;

    // the heads; the part of the keys and the unit of queries that go with it, or this wavefront's unit of queries
    int hh, qb = 0;
    uint32_t v;
    if (a.own) {
        const uint32_t groups = ((uint32_t)a.V + kWaves - 1) / kWaves * (uint32_t)packs, wg = die_order(groups);
        if (wg >= groups) return;
        hh = uniform((int)(wg % (uint32_t)packs));
        v = uniform((int)(wg / (uint32_t)packs * kWaves + wave));
    } else {
        // Parts are dealt to the 8 dies one by one, and each die has all heads and units of queries of its parts, which read the same lines.
        const uint32_t wg = blockIdx.y * gridDim.x + blockIdx.x, each = (uint32_t)packs * a.qblocks, n = wg >> 3, turn = n / each, rest = n - turn * each;
        v = uniform((int)(turn * 8 + (wg & 7u)));
        hh = uniform((int)(rest % (uint32_t)packs));
        qb = uniform((int)(rest / (uint32_t)packs));
        if (v >= (uint32_t)a.V) return;
    }
    const int head0 = hh * a.pack;
    if (BIAS) {
        fill_bias(tab, a, head0, a.pack, 64 * kWaves);
        __syncthreads();
    }
    if (v >= (uint32_t)a.V) return;
    const bool looks = hh == 0 && qb == 0 && (a.own || wave == 0) && v < (uint32_t)a.N;
    const int64_t peek = looks ? sequence_numbers(a, v) : 0;
    Sequence q;
    PartWork w;
    int part = 0;
    if (a.own) {
        const int s = find_sequence(a.q_off, a.N, v, a.block);
        const bool fits = take_sequence(a, s, sequence_numbers(a, s), q);
        const uint32_t start = (uint32_t)q.q0 / a.block + s, blocks = ((uint32_t)q.nq + a.block - 1) / a.block;
        if (!fits || v < start || v - start >= blocks) return judge(a, looks, v, peek);
        w.block = uniform((int)(v - start));
        w.blocks = w.block + 1;
        w.step = w.parts = 1;
        w.lo = 0;
        w.hi = q.nk;
    } else {
        const int s = find_part(a.k_off, a.N, v, a.cut_log2);
        const bool fits = take_sequence(a, s, sequence_numbers(a, s), q);
        const int64_t n = (int64_t)v - (s + (q.k0 >> a.cut_log2));
        part = uniform((int)n);
        if (!fits || n < 0 || n > q.nk || !part_work(a, q, part, qb, w)) return judge(a, looks, v, peek);
    }

    const int kvh = head0 / a.group;
    const char* const kb = a.k.at(q.k0, kvh);
    const char* const vb = a.v.at(q.k0, kvh);
    const float* const ks = a.ks + (int64_t)kvh * a.k_rows + q.k0;
    const float* const vs = a.vs + (int64_t)kvh * a.k_rows + q.k0;
    const int own = wave * kTile, own_scales = wave * 2 * BK, ci = col / a.pack, cg = col - ci * a.pack, head = head0 + cg;
    const int t_step = a.own ? 1 : kWaves;
    float beyond = 0.f, ahead = 0.f;
    const float* const ht = tab + cg * tab_size(a.far);
    if (BIAS) {
        beyond = ht[kTabMargin];
        ahead = a.causal ? 0.f : ht[2 * a.far + kTabMargin];
    }

    for (int block = w.block; block < w.blocks; block += w.step) {
        const int iw = block * a.block, i = iw + ci;
        const bool is = ci < a.qpt && i < q.nq;
        const int first = q.nk - q.nq + iw, pos = first + ci, wave_last = first + a.qpt - 1;   // places among the keys
        int jend = w.hi;   // keys of this unit: all that its last query sees
        if (a.causal) {
            const int last = q.nk - q.nq + (iw + a.block < q.nq ? iw + a.block : q.nq);
            jend = jend < last ? jend : last;
        }
        // this wavefront's tiles: every one, or every fourth
        const int tiles = jend > w.lo ? (jend - w.lo + BK - 1) / BK : 0, t0 = a.own ? 0 : wave;

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
        float m, sum;
        auto begin = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int d = 0; d < kD; ++d) o[d] = f32x16_t{};
            m = -__builtin_inff();
            sum = 0.f;
        };
        auto fetch = [&](const int t, char* const kt, char* const vt, float* const st) __attribute__((always_inline)) {
            const int j0 = w.lo + t * BK;
            Codes::template fetch<BK>(kt + own, kb, a.k.row, j0, q.nk, a.dim, lane);
            Codes::template fetch<BK>(vt + own, vb, a.v.row, j0, q.nk, a.dim, lane);
#pragma unroll
            for (int n = 0; n < 2 * BK / 64; ++n) {
                const int at = 64 * n + lane, j = j0 + (at & (BK - 1));
                const float* const src = (at < BK ? ks : vs) + j;
                load_lds<4>(j < q.nk ? reinterpret_cast<const char*>(src) : reinterpret_cast<const char*>(&attn_zeros), st + own_scales + 64 * n);
            }
        };
        auto step = [&](const int t, const char* const kt_, const char* const vt_, const float* const st_) __attribute__((always_inline)) {
            const int j0 = w.lo + t * BK;
            const char* const kt = kt_ + own;
            const char* const vt = vt_ + own;
            const float* const st = st_ + own_scales;
            f32x16_t x[kT];
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
            float top = -__builtin_inff();
#pragma unroll
            for (int k = 0; k < kT; ++k) {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float4 s = *reinterpret_cast<const float4*>(st + 32 * k + 2 * r + 4 * half);
                    x[k][r] *= s.x; x[k][r + 1] *= s.y; x[k][r + 2] *= s.z; x[k][r + 3] *= s.w;
                }
                if (BIAS) {
                    // (a bias of -infinity hides a score that is not finite too)
                    const int j = j0 + 32 * k;
                    if (first - (j + 31) >= a.far || wave_last - j <= -a.far) {
                        const float b = first - (j + 31) >= a.far ? beyond : ahead;
#pragma unroll
                        for (int r = 0; r < 16; ++r) x[k][r] = b == -__builtin_inff() ? b : fmaf(x[k][r], a.scale2, b);
                    } else {
                        const float* const from = ht + (j + 4 * half - pos + a.far + kTabMargin);
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float b = from[8 * (r / 4) + r % 4];
                            x[k][r] = b == -__builtin_inff() ? b : fmaf(x[k][r], a.scale2, b);
                        }
                    }
                }
            }
            if (hides) {
                const int upto = a.causal && pos + 1 < q.nk ? pos + 1 : q.nk;   // the keys that this column sees end here
#pragma unroll
                for (int k = 0; k < kT; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (j0 + 32 * k + 8 * (r / 4) + 4 * half + r % 4 >= upto) x[k][r] = -__builtin_inff();
            }
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
            const float at = m == -__builtin_inff() ? 0.f : m;   // (nothing seen so far: every probability is 2^-inf = 0)
#pragma unroll
            for (int k = 0; k < kT; ++k)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float p[8];
#pragma unroll
                    for (int r = 0; r < 8; r += 4) {
                        const float4 s4 = *reinterpret_cast<const float4*>(st + BK + 32 * k + 16 * c + 2 * r + 4 * half);
                        const float s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float y = x[k][8 * c + r + e];
                            const float at_y = __builtin_amdgcn_exp2f(BIAS ? y - at : fmaf(y, a.scale2, -at));
                            sum += at_y;
                            // (a scale that is not finite must not reach a column that does not see its key)
                            p[r + e] = at_y * (y == -__builtin_inff() ? 0.f : s[e]);
                        }
                    }
                    uint4 f[kP];
                    cut<kP>(p, f);
#pragma unroll
                    for (int d = 0; d < kD; ++d) {
                        const uint2 u = Codes::down(vt, 32 * k, c, d, lane);
                        const uint4 g = codes_bf16<I8>(u.x, u.y);
#pragma unroll
                        for (int p = kP - 1; p >= 0; --p) o[d] = M::mma(g, f[p], o[d]);
                    }
                }
            settle<bf16_t>();
        };
        // Codes that are not numbers (e4m3) among the values: a column that does not see their key would get 0 times them from the matrix cores.  They
        // are taken out of the tile, and the columns that see the key get NaN where they stood.
        auto take_out = [&](const int t) __attribute__((always_inline)) {
            const int j0 = w.lo + t * BK;
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
#pragma unroll
                for (int d = 0; d < kD; ++d)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const int e = 32 * d + 8 * n + 4 * half;
                        const uint32_t u = *reinterpret_cast<const uint32_t*>(vt + Codes::place(j, e / 16) + e % 16);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            o[d][4 * n + k] = sees && (u >> (8 * k) & 0x7Fu) == 0x7Fu ? __builtin_nanf("") : o[d][4 * n + k];
                    }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
            for (int n = lane; n < kTile / 4; n += 64) {
                uint32_t u = *reinterpret_cast<const uint32_t*>(vt + 4 * n);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if ((u >> (8 * k) & 0x7Fu) == 0x7Fu) u &= ~(0xFFu << (8 * k));
                *reinterpret_cast<uint32_t*>(vt + 4 * n) = u;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        };

        begin();
        if (t0 < tiles) fetch(t0, keys0, values0, scales0);
        for (int t = t0; t < tiles; t += 2 * t_step) {
            loads_done();
            if (t + t_step < tiles) fetch(t + t_step, keys1, values1, scales1);
            step(t, keys0, values0, scales0);
            if (t + t_step < tiles) {
                loads_done();
                if (t + 2 * t_step < tiles) fetch(t + 2 * t_step, keys0, values0, scales0);
                step(t + t_step, keys1, values1, scales1);
            }
        }
        if (!I8 && (a.causal || BIAS) && __any(is && not_finite(o))) {
            begin();
#pragma unroll 1
            for (int t = t0; t < tiles; t += t_step) {
                fetch(t, keys0, values0, scales0);
                loads_done();
                take_out(t);
                step(t, keys0, values0, scales0);
            }
        }
        sum = pair_sum<32>(sum);

        if (a.own) {
            if (is) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (no key seen: zeros)
                char* const to = const_cast<char*>(a.o.at(q.q0 + i, head));
#pragma unroll
                for (int d = 0; d < kD; ++d)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const int e = 32 * d + 2 * r + 4 * half;
                        if (e < a.dim) {
                            if constexpr (sizeof(T) == 2)
                                *reinterpret_cast<uint2*>(to + 2 * e) = make_uint2(pack2((const T*)nullptr, o[d][r] * inv, o[d][r + 1] * inv),
                                                                                   pack2((const T*)nullptr, o[d][r + 2] * inv, o[d][r + 3] * inv));
                            else *reinterpret_cast<float4*>(to + 4 * e) = make_float4(o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv);
                        }
                    }
                if (a.lse && half == 0) a.lse[(int64_t)head * a.q_rows + q.q0 + i] = sum == 0.f ? -__builtin_inff() : fmaf(m, kLn2, logf(sum));
            }
            continue;
        }
        // The wavefronts' results meet where the tiles were, as fp32 rows of D elements, sixteen bytes of a row at place c ^ column: a column's
        // lanes do not all fall on the same banks.
        auto piece = [&](const int n) __attribute__((always_inline)) { return n == 0 ? keys0 : (n == 1 ? keys1 : (n == 2 ? values0 : values1)); };
        __syncthreads();
        {
            char* const to = piece(wave);
#pragma unroll
            for (int d = 0; d < kD; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<float4*>(to + (col * kRow + ((8 * d + r / 2 + half) ^ (col % kRow))) * 16) = make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
            if (half == 0) stats[wave * 32 + col] = make_float2(m, sum);
        }
        __syncthreads();
        for (int n = threadIdx.x; n < 32 * kRow; n += 64 * kWaves) {
            const int c = n / kRow, e = n % kRow, cc = c / a.pack, ii = iw + cc, hd = head0 + c - cc * a.pack;
            if (cc >= a.qpt || ii >= q.nq) continue;
            float top = -__builtin_inff(), total = 0.f;
#pragma unroll
            for (int k = 0; k < kWaves; ++k) top = fmaxf(top, stats[k * 32 + c].x);
            const float at = top == -__builtin_inff() ? 0.f : top;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                const float2 ms = stats[k * 32 + c];
                const float by = __builtin_amdgcn_exp2f(ms.x - at);
                const float4 y = *reinterpret_cast<const float4*>(piece(k) + (c * kRow + (e ^ (c % kRow))) * 16);
                total = fmaf(ms.y, by, total);
                x.x = fmaf(y.x, by, x.x); x.y = fmaf(y.y, by, x.y);
                x.z = fmaf(y.z, by, x.z); x.w = fmaf(y.w, by, x.w);
            }
            if (w.parts > 1) {
                const int64_t cell = (((int64_t)v * a.qblocks + qb) * packs + hh) * 32 + c;
                if (e == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * cell) = make_float2(top, total);
                *reinterpret_cast<float4*>(a.part_o + cell * D + 4 * e) = x;
                continue;
            }
            const float inv = total == 0.f ? 0.f : 1.f / total;
            if (4 * e < a.dim) {
                char* const to = const_cast<char*>(a.o.at(q.q0 + ii, hd)) + 4 * e * sizeof(T);
                if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack2((const T*)nullptr, x.x * inv, x.y * inv), pack2((const T*)nullptr, x.z * inv, x.w * inv));
                else *reinterpret_cast<float4*>(to) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
            }
            if (a.lse && e == 0) a.lse[(int64_t)hd * a.q_rows + q.q0 + ii] = total == 0.f ? -__builtin_inff() : fmaf(top, kLn2, logf(total));
        }
        __syncthreads();   // (the next unit's tiles go where these results are)
    }
    judge(a, looks, v, peek);
}

// Joins the parts of the keys: a workgroup per query and head, its four wavefronts a quarter of the parts each; the order of the additions is fixed.
template <typename T, int D>
__global__ __launch_bounds__(256) void cache_attn_join_kernel(const CacheAttnArgs a) {
    constexpr int kPer = D >= 64 ? D / 64 : 1, kAhead = 8;   // elements a lane; parts under way together
    typedef float out_t __attribute__((ext_vector_type(kPer)));
    __shared__ float2 stats[4];
    __shared__ out_t sums[4][64];
    const int lane = lane_id(), wave = uniform(threadIdx.x >> 6), packs = a.H / a.pack;
    const uint32_t n = blockIdx.y * gridDim.x + blockIdx.x;
    const int64_t row = n / (uint32_t)a.H;
    const int head = (int)(n - (uint32_t)row * (uint32_t)a.H);
    if (row >= a.q_rows) return;
    const int s = find_row(a.q_off, a.N, row);
    Sequence q;
    if (!take_sequence(a, s, sequence_numbers(a, s), q) || row < q.q0 || row >= q.q0 + q.nq) return;
    const int i = (int)(row - q.q0), qb = i / a.block, blocks = (int)(((int64_t)q.nq + a.block - 1) / a.block), count = part_count(a, q.nk);
    if (blocks > a.qblocks || count < 2) return;   // (the result is there already)
    const int hh = head / a.pack, col = (i - qb * a.block) * a.pack + head - hh * a.pack;
    const int64_t each = (int64_t)a.qblocks * packs * 32;   // cells of a part
    const int64_t cell0 = (s + (q.k0 >> a.cut_log2)) * each + ((int64_t)qb * packs + hh) * 32 + col;
    const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + cell0;
    const int quarter = (count + 3) / 4, p0 = wave * quarter, p1 = p0 + quarter < count ? p0 + quarter : count;
    float m = -__builtin_inff(), sum = 0.f;
    for (int p = p0 + lane; p < p1; p += 64) m = fmaxf(m, ml[p * each].x);
#pragma unroll
    for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    const float at = m == -__builtin_inff() ? 0.f : m;
    out_t o = {};
    const int e0 = (lane * kPer) & (D - 1);   // (rows of 32 elements: the upper half of the wavefront does the same again)
    for (int base = p0; base < p1; base += 64) {
        const bool mine = base + lane < p1;
        const float2 c = mine ? ml[(base + lane) * each] : make_float2(-__builtin_inff(), 0.f);
        const float by = mine ? __builtin_amdgcn_exp2f(c.x - at) : 0.f;
        sum += group_sum(c.y * by, 64);
        const int end = p1 - base < 64 ? p1 - base : 64;
        const float* const from = a.part_o + (cell0 + base * each) * D + e0;
        for (int k = 0; k < end; k += kAhead) {
            out_t x[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) x[j] = *reinterpret_cast<const out_t*>(from + (int64_t)(k + j < end ? k + j : k) * each * D);
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (k + j < end) o += bcast_lane(by, (k + j) & 63) * x[j];
        }
    }
    if (lane == 0) stats[wave] = make_float2(m, sum);
    sums[wave][lane] = o;
    __syncthreads();
    if (wave != 0) return;
    float top = -__builtin_inff(), total = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) top = fmaxf(top, stats[k].x);
    const float all = top == -__builtin_inff() ? 0.f : top;
    out_t x = {};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float by = __builtin_amdgcn_exp2f(stats[k].x - all);
        total = fmaf(stats[k].y, by, total);
        x += by * sums[k][lane];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    T* const to = reinterpret_cast<T*>(const_cast<char*>(a.o.at(row, head)));
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e0 + e < a.dim) to[e0 + e] = elem_round<T>((kPer == 1 ? x[0] : x[e]) * inv);
    if (a.lse && lane == 0) a.lse[(int64_t)head * a.q_rows + row] = total == 0.f ? -__builtin_inff() : fmaf(top, kLn2, logf(total));
}

// How the work is shared out.  Heads of a group lie side by side in a wavefront's columns where one query would leave them empty.  Short caches, or
// so many units of queries that the chip is full: a wavefront for each unit.  Otherwise the four wavefronts of a workgroup have the same columns and
// every fourth tile of a part of the keys, joined in LDS; parts are cut so that there are at least kPartGroups workgroups.
constexpr int64_t kPartGroups = 2048;
CacheAttnPlan cache_attn_plan(const AttnShape& sh, const int max_pack) {
    CacheAttnPlan p;
    const int64_t mean_q = (sh.q_rows + sh.N - 1) / sh.N, mean_k = (sh.k_rows + sh.N - 1) / sh.N;
    p.D = sh.dim <= 32 ? 32 : (sh.dim <= 64 ? 64 : 128);
    p.pack = 1;
    const int group = sh.H / sh.kv;
    const int64_t table = sh.buckets ? (2 * (int64_t)sh.far + 1 + 2 * kTabMargin) * 4 : 0;
    for (int g = 2; g <= group && g <= max_pack; ++g)   // more heads side by side as long as a sequence's queries of all of them fit
        if (group % g == 0 && mean_q * g <= 32 && g * table <= kTabBytes) p.pack = g;
    p.block = 32 / p.pack;
    const int64_t packs = sh.H / p.pack, units = (sh.q_rows / p.block + sh.N) * packs;
    p.own = mean_k <= 128 || (units >= 4096 && mean_k <= 2048);
    p.cut_log2 = 32;
    p.qblocks = 1;
    p.V = sh.q_rows / p.block + sh.N;
    p.part_ml = p.part_o = 0;
    if (p.own) return p;
    // units of queries of a sequence that go with each part: of all sequences that are not much longer than the average
    p.qblocks = (int)std::max<int64_t>(1, (mean_q + mean_q / 4 + p.block - 1) / p.block);
    const int64_t each = packs * p.qblocks;
    p.V = sh.N;
    for (int c = 31; c >= 8; --c) {
        if (p.V * each >= kPartGroups) break;
        p.cut_log2 = c;
        p.V = (sh.k_rows >> c) + sh.N;
    }
    const int64_t cells = p.cut_log2 < 32 ? p.V * each * 32 : 0;
    p.part_ml = ((size_t)cells * 8 + 255) & ~(size_t)255;
    p.part_o = ((size_t)cells * p.D * 4 + 255) & ~(size_t)255;
    return p;
}
bool cache_attn_grid_ok(const AttnShape& sh, const CacheAttnPlan& p) {
    const int64_t most = ((int64_t)1 << 31) - 64, packs = sh.H / p.pack;
    return p.own ? (p.V + 3) / 4 * packs < most : (p.V + 7) / 8 * 8 * packs * p.qblocks < most && (p.part_ml == 0 || sh.q_rows * sh.H < most);
}
size_t cache_attn_workspace(const AttnShape& sh) {
    size_t most = 0;
    for (int pack = 1; pack <= 32; ++pack) {   // (how many heads go side by side depends on the bias)
        AttnShape any = sh;
        any.far = 0;
        const CacheAttnPlan p = cache_attn_plan(any, pack);
        most = std::max(most, p.part_ml + p.part_o);
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
static hipError_t launch_dim(const tbe_handle* h, const CacheAttnArgs& a, const bool i8, const uint64_t groups, const bool join, hipStream_t s) {
    const hipError_t e = i8 ? launch_parts<T, D, true>(h, a, groups, s) : launch_parts<T, D, false>(h, a, groups, s);
    if (e != hipSuccess || !join) return e;
    LaunchTimer tm(h, s, "cache_attention_join");
    cache_attn_join_kernel<T, D><<<die_grid((uint64_t)a.q_rows * (uint64_t)a.H), 256, 0, s>>>(a);
    tm.done();
    return hipGetLastError();
}
template <typename T>
static hipError_t launch_type(const tbe_handle* h, const CacheAttnArgs& a, const int D, const bool i8, const uint64_t groups, const bool join, hipStream_t s) {
    return D == 32 ? launch_dim<T, 32>(h, a, i8, groups, join, s) : (D == 64 ? launch_dim<T, 64>(h, a, i8, groups, join, s) : launch_dim<T, 128>(h, a, i8, groups, join, s));
}

hipError_t launch_cache_attention(const tbe_handle* h, const AttnArgs& call, const CodeRows (&cache)[2], const bool i8, const CacheAttnPlan& p, const int io,
                                  void* workspace, hipStream_t s) {
    CacheAttnArgs a{};
    static_cast<AttnArgs&>(a) = call;
    a.k = cache[0].codes; a.v = cache[1].codes;
    a.ks = cache[0].scales; a.vs = cache[1].scales;
    a.pack = p.pack; a.qpt = a.block = p.block; a.V = (int)p.V;
    a.cut_log2 = p.cut_log2; a.qblocks = p.qblocks; a.own = p.own;
    a.part_ml = static_cast<float*>(workspace);
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_ml);
    const uint64_t packs = (uint64_t)(a.H / a.pack);
    const uint64_t groups = p.own ? ((uint64_t)p.V + 3) / 4 * packs : ((uint64_t)p.V + 7) / 8 * 8 * packs * (uint64_t)p.qblocks;
    const bool join = p.part_ml > 0;
    return io == 0 ? launch_type<float>(h, a, p.D, i8, groups, join, s) : (io == 1 ? launch_type<__half>(h, a, p.D, i8, groups, join, s) : launch_type<bf16_t>(h, a, p.D, i8, groups, join, s));
}

}  // namespace tbe
