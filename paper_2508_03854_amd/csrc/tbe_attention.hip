// Attention over packed sequences, forward (see tbe355.h for what it computes): one pass over the keys with the running maximum and sum
// of the softmax; no score leaves the registers.
//   S^T = K Q^T  (a tile: 32 keys x 32 columns)    p = 2^(x - m)    O^T += V^T P
// Bound: long sequences by the vector unit's work on every score (the exponential, the sums) next to the matrix cores, single tokens by
// reading the keys and values once, many short sequences by a wavefront's trips to memory.  Measured: 2 causal sequences of 4000 to 8000, 16
// heads of 128 over 4, bfloat16, 2.3e11 operations: 266 us when called one after the other, 0.86 PFLOP/s, up to 313 with other work between; one
// query to each of 24 caches of 2000 to 65536 keys, 16 heads over 2, 0.8 GB: 168 us and 8 for the join, 4.6 TB/s; 4096 sequences of 12 events
// on average, 4 heads of 32 with a bias: 21 us for 51 MB.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tbe_attention.h"

namespace tbe {

// SHARE = 4: the four wavefronts of a workgroup take neighbouring queries of one head and share the tiles of keys and values.
// SHARE = 1: every wavefront is on its own, with `pack` heads of a group side by side in its columns; or (together) the wavefronts of a
// workgroup have the same columns and a part of the keys each, joined in LDS, and with splits > 1 several workgroups do, joined by
// attn_join_kernel.
// SHARE = 0: short sequences: a wavefront takes 32 neighbouring rows of q, whosesoever they are, and the keys of all their sequences; a column
// hides what is not its own sequence's (see kManyUnits).
// Rows of a tile of keys: 64 where the LDS has room for two of them of keys and of values and a second workgroup (2 sequences of 6000, 16 heads of 128
// bfloat16: 64 rows 331 us, 32 rows 363; heads of 64 172 / 169 and of 32 128 / 126 with either).
template <typename T, int D, int SHARE>
constexpr int kv_rows() { return SHARE == 4 && D * (int)sizeof(T) <= 256 ? 64 : 32; }
template <typename T, int D, int SHARE>
constexpr int attn_waves() { return SHARE != 4 && D * (int)sizeof(T) > 256 ? 2 : 4; }

template <typename T, int D, int SHARE>   // wavefronts of a SIMD that the registers are to leave room for (and the LDS does)
constexpr int attn_occupancy() { return sizeof(T) == 4 ? (D == 32 ? 2 : 1) : (D == 32 ? 4 : (D == 64 ? (SHARE == 4 ? 3 : 2) : (SHARE == 4 ? 2 : 1))); }

template <typename T, int D, int SHARE, bool BIAS>
__global__ __launch_bounds__((64 * attn_waves<T, D, SHARE>()), (attn_occupancy<T, D, SHARE>())) void attn_kernel(const AttnArgs a) {
    constexpr int kWaves = attn_waves<T, D, SHARE>(), BK = kv_rows<T, D, SHARE>(), kT = BK / 32, kD = D / 32;
    constexpr int kK = Mma<T>::kK, kC = D / kK, kM = 32 / kK;
    constexpr int kTile = BK * D * (int)sizeof(T), kSharers = SHARE == 4 ? 4 : 1;
    constexpr bool kRows = SHARE == 0;
    // two buffers each, as arrays of their own: loads into one of them are seen not to concern what is read from another
    constexpr int kLds = SHARE == 4 ? kTile : kWaves * kTile;
    __shared__ __align__(16) char keys0[kLds], keys1[kLds], values0[kLds], values1[kLds];
    __shared__ int votes[kWaves];
    extern __shared__ float tab[];
    const int wave = uniform(threadIdx.x >> 6), lane = lane_id(), col = lane & 31, half = lane >> 5;
    const bool together = SHARE == 1 && a.together;
    const uint32_t per_head = SHARE == 4 || together ? (uint32_t)a.V * a.splits : ((uint32_t)a.V + kWaves - 1) / kWaves;
    const uint32_t groups = per_head * (uint32_t)(a.H / a.pack), wg = die_order(groups);
    if (wg >= groups) return;
    int hh;
    uint32_t item;
    head_and_item<SHARE>(wg, per_head, a.H / a.pack, hh, item);
    const int head0 = hh * a.pack;
    if (BIAS) {
        fill_bias(tab, a, head0, a.pack, 64 * kWaves);
        __syncthreads();
    }
    const uint32_t unit = SHARE == 4 || together ? item : item * kWaves + wave;
    if (unit >= (uint32_t)a.V * a.splits) return;
    const uint32_t v = SHARE != 1 ? unit : unit / a.splits;
    const int split = SHARE != 1 ? 0 : unit - v * a.splits;
    const bool looks = !kRows && hh == 0 && split == 0 && ((SHARE == 1 && !together) || wave == 0) && v < (uint32_t)a.N;
    const int64_t peek = looks ? sequence_numbers(a, v) : 0;
    Sequence q;
    int i0, iw, i, cg = 0, head = head0, first, pos, jend;
    bool is;
    // SHARE = 0: this column's own keys and its place among all rows of k
    int own_lo = 0, own_end = 0, own_pos = 0;
    if constexpr (kRows) {
        if (hh == 0) judge_all(a, v, a.V);
        q.q0 = (int64_t)v * 32;
        q.k0 = 0;
        q.nk = (int)a.k_rows;
        q.nq = 32;
        const LaneSequence mine = lane_numbers(a, lane_sequence(a.q_off, a.N, q.q0, a.q_rows));
        const int64_t row = q.q0 + col;
        is = mine.fits && row >= mine.q0 && row < mine.q1;
        own_pos = (int)(mine.k1 - mine.q1 + row);
        own_lo = is ? (int)mine.k0 : 0;
        own_end = is ? (int)mine.k1 : 0;
        if (a.causal && own_pos + 1 < own_end) own_end = own_pos + 1;
        if (own_end < own_lo) own_end = own_lo;
        i0 = iw = 0;
        i = col;
        first = pos = jend = 0;
        if (!__any(is)) return;
    } else {
        const int s = find_sequence(a.q_off, a.N, v, a.block);
        const bool fits = take_sequence(a, s, sequence_numbers(a, s), q);
        const uint32_t start = (uint32_t)q.q0 / a.block + s, blocks = ((uint32_t)q.nq + a.block - 1) / a.block;
        if (!fits || v < start || v - start >= blocks) return judge(a, looks, v, peek);
        // the last queries, which see the most keys, first
        i0 = uniform((int)(blocks - 1 - (v - start)) * a.block);
        iw = i0 + (SHARE == 4 ? wave * 32 : 0);
        const int ci = SHARE == 4 ? col : col / a.pack;
        cg = SHARE == 4 ? 0 : col - ci * a.pack;
        i = iw + ci;
        head = head0 + cg;
        is = ci < a.qpt && i < q.nq;
        first = q.nk - q.nq + iw;   // place among the keys of the wavefront's first query ...
        pos = first + ci;           // ... and of this column's
        // keys of this unit: all that its last query sees
        jend = q.nk;
        if (a.causal) {
            const int last = q.nk - q.nq + (i0 + a.block < q.nq ? i0 + a.block : q.nq);
            jend = jend < last ? jend : last;
        }
    }

    uint4 fq[kC];
    column_row<T, D>(fq, a.q.at(q.q0 + (is ? i : 0), head), is, half, a.dim);
    if (a.negative) flip_signs<T, kC>(fq);
    // ... or a part of them
    int t0 = 0, t1, jbase = 0, lo = 0, end = 0;
    {
        const int tiles = jend > 0 ? (jend + BK - 1) / BK : 0;
        const int parts = together ? a.splits * kWaves : 1, part = (tiles + parts - 1) / parts;
        if (together) t0 = uniform((split * kWaves + wave) * part);
        t1 = uniform(t0 + part < tiles ? t0 + part : tiles);
    }
    int wave_last = first + a.qpt - 1;   // the last place that a query of this wavefront may have

    const int kvh = head0 / a.group;
    const char* const kb = a.k.at(q.k0, kvh);
    const char* const vb = a.v.at(q.k0, kvh);
    const int own = SHARE == 4 ? 0 : wave * kTile, fw = SHARE == 4 ? wave : 0;
    auto fetch = [&](const int t, char* const kt, char* const vt, const int l) __attribute__((always_inline)) {
        Tile<T, D>::template fetch<BK, kSharers>(kt + own, kb, a.k.row, jbase + t * BK, q.nk, a.dim, fw, l);
        Tile<T, D>::template fetch<BK, kSharers>(vt + own, vb, a.v.row, jbase + t * BK, q.nk, a.dim, fw, l);
    };

    f32x16_t o[kD];
#pragma unroll
    for (int d = 0; d < kD; ++d) o[d] = f32x16_t{};
    float m = -__builtin_inff(), sum = 0.f;
    float beyond = 0.f, ahead = 0.f;
    const float* const ht = tab + cg * tab_size(a.far);
    if (BIAS) {
        beyond = ht[kTabMargin];
        ahead = a.causal ? 0.f : ht[2 * a.far + kTabMargin];
    }

    // 32 keys from key j on: scores with their bias (as exponents of 2; without a bias they are scaled later), hidden ones at -infinity
    auto biased = [&](f32x16_t& x, const int j) __attribute__((always_inline)) {
        if (first - (j + 31) >= a.far || wave_last - j <= -a.far) {
            const float b = first - (j + 31) >= a.far ? beyond : ahead;
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], a.scale2, b);
        } else {
            const float* const from = ht + (j + 4 * half - pos + a.far + kTabMargin);
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], a.scale2, from[8 * (r / 4) + r % 4]);
        }
    };
    auto hidden = [&](f32x16_t& x, const int j) __attribute__((always_inline)) {
        if constexpr (kRows) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if ((uint32_t)(j + 8 * (r / 4) + 4 * half + r % 4 - lo) >= (uint32_t)(end - lo)) x[r] = -__builtin_inff();
        } else {
            const int upto = a.causal && pos + 1 < q.nk ? pos + 1 : q.nk;   // the keys that this column sees end here
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (j + 8 * (r / 4) + 4 * half + r % 4 >= upto) x[r] = -__builtin_inff();
        }
    };
    // A maximum that grows by less than 2^8 is left as it is: the probabilities stay below 2^8, and what they are divided by in the end is
    // added up from them.
    auto raise = [&](const float top) __attribute__((always_inline)) {
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
    };
    auto hides = [&](const int j0) { return kRows || j0 + BK > q.nk || (a.causal && j0 + BK - 1 > first); };
    auto step = [&](const int t, const char* const kt_, const char* const vt_, char* const kn, char* const vn) __attribute__((always_inline)) {
        loads_done();
        if (SHARE == 4) __syncthreads();
        if (t + 1 < t1) fetch(t + 1, kn, vn, lane);
        const int j0 = jbase + t * BK;
        const char* const kt = kt_ + own;
        const char* const vt = vt_ + own;
        if (SHARE == 4 && ((a.causal && j0 > wave_last) || iw >= q.nq)) return;
        f32x16_t x[kT];
#pragma unroll
        for (int k = 0; k < kT; ++k) {
            x[k] = f32x16_t{};
#pragma unroll
            for (int c = 0; c < kC; ++c) x[k] = Mma<T>::mma(Tile<T, D>::along(kt, 32 * k + col, c, half), fq[c], x[k]);
        }
        reads_ahead<kT * kC, 1, Mma<T>::kMfmas, 4>();
        settle<T>();
        if (BIAS) {
#pragma unroll
            for (int k = 0; k < kT; ++k) biased(x[k], j0 + 32 * k);
        }
        if (hides(j0)) {
#pragma unroll
            for (int k = 0; k < kT; ++k) hidden(x[k], j0 + 32 * k);
        }
        float top = x[0][0];
#pragma unroll
        for (int k = 0; k < kT; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, x[k][r]);
        top = halves_max(top);
        if (!BIAS) top *= a.scale2;
        raise(top);
        const float at = m == -__builtin_inff() ? 0.f : m;   // (nothing seen so far: every probability is 2^-inf = 0)
#pragma unroll
        for (int k = 0; k < kT; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[k][r] = __builtin_amdgcn_exp2f(BIAS ? x[k][r] - at : fmaf(x[k][r], a.scale2, -at));
                sum += x[k][r];
            }
        uint4 p[kT][kM];   // (rounded to the values' type: the sum they are divided by is not)
#pragma unroll
        for (int k = 0; k < kT; ++k)
#pragma unroll
            for (int c = 0; c < kM; ++c) p[k][c] = Mma<T>::pack(x[k], c);
#pragma unroll
        for (int k = 0; k < kT; ++k)
#pragma unroll
            for (int c = 0; c < kM; ++c)
#pragma unroll
                for (int d = 0; d < kD; ++d) o[d] = Mma<T>::mma(Tile<T, D>::down(vt, 32 * k, c, d), p[k][c], o[d]);
        reads_ahead<kT * kM * kD, Mma<T>::kDown, Mma<T>::kMfmas, 4>();
        settle<T>();
    };
    // The same with care for values that are not finite: their elements are multiplied one by one, for the columns that see them (see
    // Tile::cleaned).  Every number is the step's own, bit by bit; 32 keys and one tile at a time, since registers are short.
    auto careful_step = [&](const int t) __attribute__((always_inline)) {
        if (SHARE == 4) __syncthreads();
        const int l = anew(lane), c32 = l & 31, h = l >> 5;
        fetch(t, keys0, values0, l);
        loads_done();
        if (SHARE == 4) __syncthreads();
        const int j0 = jbase + t * BK;
        if (SHARE == 4 && ((a.causal && j0 > wave_last) || iw >= q.nq)) return;
        f32x16_t x;
        auto scores = [&](const int k) __attribute__((always_inline)) {
            x = f32x16_t{};
#pragma unroll
            for (int c = 0; c < kC; ++c) x = Mma<T>::mma(Tile<T, D>::along(keys0 + own, 32 * k + c32, c, h), fq[c], x);
            reads_ahead<kC, 1, Mma<T>::kMfmas, 2>();
            settle<T>();
            if (BIAS) biased(x, j0 + 32 * k);
            if (hides(j0)) hidden(x, j0 + 32 * k);
        };
        float top = -__builtin_inff();
#pragma unroll 1
        for (int k = 0; k < kT; ++k) {
            scores(k);
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, x[r]);
        }
        top = halves_max(top);
        if (!BIAS) top *= a.scale2;
        raise(top);
        const float at = m == -__builtin_inff() ? 0.f : m;
#pragma unroll 1
        for (int k = 0; k < kT; ++k) {
            const int j = j0 + 32 * k;
            scores(k);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] = __builtin_amdgcn_exp2f(BIAS ? x[r] - at : fmaf(x[r], a.scale2, -at));
                sum += x[r];
            }
            Tile<T, D>::add_not_finite(o, values0 + own, 32 * k, x, (kRows ? lo : 0) - j, (kRows ? end : (a.causal && pos + 1 < q.nk ? pos + 1 : q.nk)) - j, l);
#pragma unroll
            for (int c = 0; c < kM; ++c) {
                const uint4 p = Mma<T>::pack(x, c);
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    o[d] = Mma<T>::mma(Tile<T, D>::cleaned(Tile<T, D>::down(values0 + own, 32 * k, c, d, l)), p, o[d]);
                    __builtin_amdgcn_sched_barrier(0);   // (few registers rather than many loads under way)
                }
            }
            settle<T>();
        }
    };
    // SHARE = 0: columns whose places lie as their rows do go together: all of them where queries and keys are the same rows.
    auto take_some = [&](uint64_t& todo) __attribute__((always_inline)) {
        const int shift = uniform(bcast_lane(own_pos - col, __ffsll((unsigned long long)todo) - 1));
        const bool mine = is && own_pos - col == shift;
        todo &= ~__ballot(mine);
        first = shift;
        pos = first + col;
        wave_last = first + 31;
        lo = mine ? own_lo : 0;
        end = mine ? own_end : 0;
        jbase = wave_min_i32(lo < end ? lo : 0x7FFFFFFF);
        const int last = wave_max_i32(lo < end ? end : 0);
        t1 = jbase < last ? (last - jbase + BK - 1) / BK : 0;
    };
    for (uint64_t todo = kRows ? __ballot(is) : 1; todo;) {
        if constexpr (kRows) take_some(todo);
        else todo = 0;
        if (t0 < t1) fetch(t0, keys0, values0, lane);
        for (int t = t0; t < t1; t += 2) {
            step(t, keys0, values0, keys1, values1);
            if (t + 1 < t1) step(t + 1, keys1, values1, keys0, values0);
        }
    }
    // The probability of a hidden key is 0, but 0 times a value that is not finite is not: where some keys are hidden and a result is not finite, all is
    // done once more (see Tile::cleaned).  Who shares tiles runs together.
    if ((kRows || a.causal) && any_sharer<SHARE>(is && not_finite(o), votes, wave)) {
#pragma unroll
        for (int d = 0; d < kD; ++d) o[d] = f32x16_t{};
        m = -__builtin_inff();
        sum = 0.f;
        for (uint64_t todo = kRows ? __ballot(is) : 1; todo;) {
            if constexpr (kRows) take_some(todo);
            else todo = 0;
#pragma unroll 1
            for (int t = t0; t < t1; ++t) careful_step(t);
        }
    }
    if (!kRows) judge(a, looks, v, peek);
    sum = pair_sum<32>(sum);
    if (SHARE == 1 && together) {
        // The parts' results meet where the tiles were, as fp32 rows of D elements, sixteen bytes of a row at place c ^ column: a column's
        // lanes do not all fall on the same banks.
        constexpr int kRow = D / 4;
        auto piece = [&](const int w) __attribute__((always_inline)) {
            return sizeof(T) == 2 ? (w < 2 ? keys0 : keys1) + (w & 1) * 128 * D : keys0 + w * 128 * D;
        };
        __shared__ float2 stats[kWaves * 32];
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
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stats[w * 32 + c].x);
            const float at = top == -__builtin_inff() ? 0.f : top;
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float2 ms = stats[w * 32 + c];
                const float by = __builtin_amdgcn_exp2f(ms.x - at);
                const float4 y = *reinterpret_cast<const float4*>(piece(w) + (c * kRow + (e ^ (c % kRow))) * 16);
                total = fmaf(ms.y, by, total);
                x.x = fmaf(y.x, by, x.x); x.y = fmaf(y.y, by, x.y);
                x.z = fmaf(y.z, by, x.z); x.w = fmaf(y.w, by, x.w);
            }
            if (a.splits > 1) {
                const int64_t cell = (((int64_t)hh * a.V + v) * a.splits + split) * 32 + c;
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
        return;
    }
    if (!is) return;
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

// Joins the parts of the keys: one wavefront per query and head, in the order of the parts.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(const AttnArgs a) {
    const int lane = lane_id();
    const int64_t n = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = (int)(n & 31);
    const int64_t hv = n >> 5;
    const int hh = (int)(hv / a.V), ci = col / a.pack, head = hh * a.pack + col - ci * a.pack;
    const uint32_t v = (uint32_t)(hv - (int64_t)hh * a.V);
    if (hh >= a.H / a.pack || ci >= a.qpt) return;
    const int s = find_sequence(a.q_off, a.N, v, a.block);
    Sequence q;
    if (!take_sequence(a, s, sequence_numbers(a, s), q)) return;
    const uint32_t start = (uint32_t)q.q0 / a.block + s, blocks = ((uint32_t)q.nq + a.block - 1) / a.block;
    if (v < start || v - start >= blocks) return;
    const int i = (int)(blocks - 1 - (v - start)) * a.block + ci;
    if (i >= q.nq) return;
    // lane k: the maximum, sum and weight of parts k and k + 64 (there are at most 128)
    const int64_t p0 = hv * a.splits * 32 + col;
    const float2 none = make_float2(-__builtin_inff(), 0.f);
    const float2 ml0 = lane < a.splits ? *reinterpret_cast<const float2*>(a.part_ml + 2 * (p0 + 32 * lane)) : none;
    const float2 ml1 = lane + 64 < a.splits ? *reinterpret_cast<const float2*>(a.part_ml + 2 * (p0 + 32 * (lane + 64))) : none;
    float m = fmaxf(ml0.x, ml1.x);
#pragma unroll
    for (int w = 32; w; w >>= 1) m = fmaxf(m, __shfl_xor(m, w));
    const float at = m == -__builtin_inff() ? 0.f : m;
    const float w0 = __builtin_amdgcn_exp2f(ml0.x - at), w1 = __builtin_amdgcn_exp2f(ml1.x - at);
    const float sum = group_sum(fmaf(ml0.y, w0, ml1.y * w1), 64);
    constexpr int kPer = D >= 64 ? D / 64 : 1, kAhead = 8;   // elements a lane; parts under way together
    typedef float out_t __attribute__((ext_vector_type(kPer)));
    out_t o = {};
    const int e0 = (lane * kPer) & (D - 1);   // (rows of 32 elements: the upper half of the wavefront does the same again)
    const float* const from = a.part_o + p0 * D + e0;
    for (int k = 0; k < a.splits; k += kAhead) {
        out_t x[kAhead];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) x[n] = *reinterpret_cast<const out_t*>(from + (int64_t)(k + n < a.splits ? k + n : k) * 32 * D);
#pragma unroll
        for (int n = 0; n < kAhead; ++n)
            if (k + n < a.splits) o += bcast_lane(k + n < 64 ? w0 : w1, (k + n) & 63) * x[n];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T* const to = reinterpret_cast<T*>(const_cast<char*>(a.o.at(q.q0 + i, head)));
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e0 + e < a.dim) to[e0 + e] = elem_round<T>((kPer == 1 ? o[0] : o[e]) * inv);
    if (a.lse && lane == 0) a.lse[(int64_t)head * a.q_rows + q.q0 + i] = sum == 0.f ? -__builtin_inff() : fmaf(m, kLn2, logf(sum));
}

// How the forward shares out its work.  Sequences of many queries: 128 neighbours share the keys' tiles (see attn_few).  Few queries per
// sequence: wavefronts on their own, heads of a group side by side where one query would leave its columns empty (24 caches of 34,000 keys, one
// query, 16 heads of 2: 178 us; one head each: 922), and the keys in parts of 128 or more where there would be fewer than 2048 wavefronts.  Parts
// for one query of 16 heads of 2 of 128 elements, none / this, us with the join: one cache of 256 keys 16.4 / 11.4, of 16,384 471 / 23; 64 of them 644 /
// 195; for half as many wavefronts 191 (but 61 queries each of 8 heads of 64 112 / 63), for twice as many 204; parts of 64 or more keys, one cache
// of 256, 1024, 16,384 keys: 11.5 / 11.4, 19 / 20, 25 / 23; of 256 or more 16 / 11, 17 / 20, 25 / 23.
AttnPlan attn_plan(const AttnShape& sh, const int max_pack) {
    AttnPlan p;
    const int64_t mean_q = sh.N > 0 ? (sh.q_rows + sh.N - 1) / sh.N : 0, mean_k = sh.N > 0 ? (sh.k_rows + sh.N - 1) / sh.N : 0;
    p.D = sh.dim <= 32 ? 32 : (sh.dim <= 64 ? 64 : 128);
    p.pack = 1;
    p.splits = 1;
    p.shared = !attn_few(mean_q, mean_k, p.D == 32 ? 128 : (p.D == 64 ? 256 : 64));
    if (p.shared) {
        p.qpt = 32;
        p.block = 128;
    } else {
        const int group = sh.H / sh.kv;
        const int64_t table = sh.buckets ? (2 * (int64_t)sh.far + 1 + 2 * kTabMargin) * 4 : 0;
        for (int g = 2; g <= group && g <= max_pack; ++g)   // more heads side by side as long as a sequence's queries of all of them fit
            if (group % g == 0 && mean_q * g <= 32 && g * table <= kTabBytes) p.pack = g;
        p.qpt = p.block = 32 / p.pack;
    }
    p.rows = !p.shared && p.pack == 1 && !sh.caches && mean_k <= 2 * mean_q && (sh.q_rows / 32 + sh.N) * sh.H >= kManyUnits;
    p.V = p.rows ? (sh.q_rows + 31) / 32 : sh.q_rows / p.block + sh.N;
    p.together = false;
    if (!p.shared) {
        const int64_t units = (sh.q_rows / p.block < sh.N ? sh.N : sh.q_rows / p.block + sh.N / 2) * (sh.H / p.pack);
        const int64_t want = p.rows ? 1 : std::min(units > 0 ? 2048 / units : 1, mean_k / 128);
        p.together = want > 1;
        p.splits = (int)std::min<int64_t>(128, std::max<int64_t>(1, (want + 3) / 4));
    }
    const int64_t cells = (int64_t)(sh.H / p.pack) * p.V * p.splits * 32;
    p.part_ml = p.splits > 1 ? ((size_t)cells * 8 + 255) & ~(size_t)255 : 0;
    p.part_o = p.splits > 1 ? ((size_t)cells * p.D * 4 + 255) & ~(size_t)255 : 0;
    return p;
}

bool attn_grid_ok(const AttnShape& sh, const AttnPlan& p) {
    return (int64_t)(sh.H / p.pack) * p.V * (p.splits > 1 ? 8 * (int64_t)p.splits : 1) < ((int64_t)1 << 31) - 64;
}
size_t attn_workspace(const AttnShape& sh, const bool backward) {
    if (backward) return attn_backward_workspace(sh);
    size_t most = 0;
    for (int pack = 1; pack <= 32; ++pack) {   // (how many heads go side by side depends on the bias)
        AttnShape any = sh;
        any.far = 0;
        any.caches = true;
        const AttnPlan p = attn_plan(any, pack);
        most = std::max(most, p.part_ml + p.part_o);
    }
    return most;
}

template <typename T, int D, int SHARE, bool BIAS>
static hipError_t launch_one(const AttnArgs& a, hipStream_t s) {
    constexpr int kWaves = attn_waves<T, D, SHARE>();
    const size_t table = BIAS ? (size_t)a.pack * (2 * a.far + 1 + 2 * kTabMargin) * 4 : 0;
    const uint64_t per_head = SHARE == 4 || a.together ? (uint64_t)a.V * a.splits : ((uint64_t)a.V + kWaves - 1) / kWaves;
    const uint64_t groups = per_head * (uint64_t)(a.H / a.pack);
    attn_kernel<T, D, SHARE, BIAS><<<die_grid(groups), 64 * kWaves, table, s>>>(a);
    return hipGetLastError();
}
template <typename T, int D>
static hipError_t launch_dim(const tbe_handle* h, const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    hipError_t e;
    {
        LaunchTimer tm(h, s, "attention");
        if (p.shared) e = a.bias ? launch_one<T, D, 4, true>(a, s) : launch_one<T, D, 4, false>(a, s);
        else if (p.rows) e = a.bias ? launch_one<T, D, 0, true>(a, s) : launch_one<T, D, 0, false>(a, s);
        else e = a.bias ? launch_one<T, D, 1, true>(a, s) : launch_one<T, D, 1, false>(a, s);
        tm.done();
    }
    if (e != hipSuccess || p.splits == 1) return e;
    LaunchTimer tm(h, s, "attention_join");
    attn_join_kernel<T, D><<<(unsigned)((int64_t)(a.H / a.pack) * a.V * 8), 256, 0, s>>>(a);
    tm.done();
    return hipGetLastError();
}
template <typename T>
static hipError_t launch_type(const tbe_handle* h, const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    return p.D == 32 ? launch_dim<T, 32>(h, a, p, s) : (p.D == 64 ? launch_dim<T, 64>(h, a, p, s) : launch_dim<T, 128>(h, a, p, s));
}

hipError_t launch_attention(const tbe_handle* h, AttnArgs a, const AttnPlan& p, int io, void* workspace, hipStream_t s) {
    a.pack = p.pack; a.qpt = p.qpt; a.block = p.block; a.V = (int)p.V; a.splits = p.splits; a.together = p.together;
    a.part_ml = static_cast<float*>(workspace);
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_ml);
    return io == 0 ? launch_type<float>(h, a, p, s) : (io == 1 ? launch_type<__half>(h, a, p, s) : launch_type<bf16_t>(h, a, p, s));
}

}  // namespace tbe
