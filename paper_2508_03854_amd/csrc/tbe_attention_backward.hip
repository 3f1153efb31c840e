// Gradients of attention over packed sequences (see tbe355.h).  The scores are computed again from q and k, the probabilities from them and
// the forward's lse; two kernels, so that every sum has one owner and a fixed order:
//   attn_dq_kernel    columns are queries:  S^T = K Q^T, dP^T = V dO^T, dS;  dQ^T += K^T dS;  also D = rowsum(dO O), and dbias
//   attn_dkv_kernel   columns are keys:     S = Q K^T,   dP = dO V^T,   dS;  dV^T += dO^T P,  dK^T += Q^T dS
// Seven products of a tile instead of five: sums of dQ from one kernel over key blocks would need atomics or a pass over partial sums.
// Bound: the matrix cores and the vector unit's work on every score, twice; short sequences by the trips to memory of a wavefront.  Measured: 4
// causal sequences of 1000 to 4096, 8 heads of 64 over 2, binary16, a bias of 32 buckets, 6.0e10 operations: dq 129, dbias 5, dk and dv 134 and
// their join 8 us, 0.22 PFLOP/s; 4096 sequences of 12
// events on average, 4 heads of 32: 57 + 5 + 39 us for 103 MB.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tbe_attention.h"

namespace tbe {

static __device__ const float attn_inf = __builtin_inff();

// SHARE = 4: the wavefronts of a workgroup take neighbouring columns of one sequence and share tiles.  SHARE = 1: each is on its own.
// SHARE = 0: each is on its own and takes 32 neighbouring rows, whosesoever they are, with all that their sequences have on the other
// side; a column hides what is not its own sequence's (see kManyUnits).
template <typename T, int D, int SHARE>
constexpr int bwd_rows() { return SHARE == 4 && D * (int)sizeof(T) <= 128 ? 64 : 32; }
template <typename T, int D, int SHARE>
constexpr int bwd_waves() { return SHARE == 4 ? 4 : (D * (int)sizeof(T) <= 128 ? 4 : (D * (int)sizeof(T) <= 256 ? 2 : 1)); }
template <typename T, int D, int SHARE>   // wavefronts of a SIMD that the registers are to leave room for
constexpr int dq_occupancy() { return sizeof(T) == 2 && (D <= 64 || SHARE == 4) ? 2 : 1; }
template <typename T, int D>
constexpr int dkv_occupancy() { return sizeof(T) == 2 ? (D == 32 ? 3 : (D == 64 ? 2 : 1)) : 1; }

// a column's share of a transposed result, times `by`, to its row
template <typename T, int D>
__device__ __forceinline__ void store_column(char* row, const f32x16_t (&o)[D / 32], const float by, const int half, const int dim) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int e = 32 * d + 2 * r + 4 * half;
            if (e < dim) {
                if constexpr (sizeof(T) == 2)
                    *reinterpret_cast<uint2*>(row + 2 * e) = make_uint2(pack2((const T*)nullptr, o[d][r] * by, o[d][r + 1] * by),
                                                                        pack2((const T*)nullptr, o[d][r + 2] * by, o[d][r + 3] * by));
                else *reinterpret_cast<float4*>(row + 4 * e) = make_float4(o[d][r] * by, o[d][r + 1] * by, o[d][r + 2] * by, o[d][r + 3] * by);
            }
        }
}

// Sums along the diagonals of a tile of 32 keys (rows: registers) by 32 queries (columns: lanes): lane `col` of a half gets, for that half's
// rows, which begin at 4 * half, the sums for key - query = 4 half - col (first) and 32 + 4 half - col (second).
// Row 16 c + n of the tile moved n lanes down its 16-lane row has one diagonal per lane, but for the lanes that it leaves, which are the
// ends of the next diagonals 16 away: a shift one way and the other, each part of an addition.  No trip through the LDS: one
// addition to an LDS word per value took 215 clocks for a wavefront's 64.
template <int R>
__device__ __forceinline__ void diagonal_row(const f32x16_t& g, float (&d)[3]) {
    constexpr int n = 8 * ((R / 4) % 2) + R % 4, c = R / 8;
    if constexpr (n == 0) {
        d[c] += g[R];
    } else {
        d[c] += dpp_lane<0x100 + n>(g[R]);            // row_shl:n, zeros from beyond
        d[c + 1] += dpp_lane<0x110 + 16 - n>(g[R]);   // row_shr:16-n
    }
}
__device__ __forceinline__ float2 diagonal_sums(const f32x16_t& g) {
    float d[3] = {0.f, 0.f, 0.f};   // key - query = 4 half + 16 (i - lane row) - lane in row
    diagonal_row<0>(g, d); diagonal_row<1>(g, d); diagonal_row<2>(g, d); diagonal_row<3>(g, d);
    diagonal_row<4>(g, d); diagonal_row<5>(g, d); diagonal_row<6>(g, d); diagonal_row<7>(g, d);
    diagonal_row<8>(g, d); diagonal_row<9>(g, d); diagonal_row<10>(g, d); diagonal_row<11>(g, d);
    diagonal_row<12>(g, d); diagonal_row<13>(g, d); diagonal_row<14>(g, d); diagonal_row<15>(g, d);
    const unsigned u = __float_as_uint(d[1]);
    const auto rows = __builtin_amdgcn_permlane16_swap(u, u, false, false);   // the even and the odd row's d[1], each in both
    const bool odd = lane_id() & 16;
    return make_float2(d[0] + (odd ? 0.f : __uint_as_float(rows[1])), d[2] + (odd ? __uint_as_float(rows[0]) : 0.f));
}

// dbias of a unit: its sums by distance, [from, to) of a table, added up by bucket; `lane` of `lanes` does every lanes-th bucket.
// bucket: the bucket of every entry of the table.
__device__ __forceinline__ void bucket_sums(const AttnArgs& a, float* out, const float* sums, const uint16_t* bucket, const int from, const int to,
                                            const float beyond, const float ahead, const int lane, const int lanes) {
    const int b_beyond = bucket[kTabMargin], b_ahead = bucket[2 * a.far + kTabMargin];
    for (int b = lane; b < a.buckets; b += lanes) {
        float s = (b == b_beyond ? beyond : 0.f) + (!a.causal && b == b_ahead ? ahead : 0.f);
#pragma unroll 8
        for (int t = from; t < to; ++t) s += bucket[t] == b ? sums[t] : 0.f;
        out[b] = s;
    }
}

template <typename T, int D, int SHARE, bool BIAS>
__global__ __launch_bounds__((64 * bwd_waves<T, D, SHARE>()), (dq_occupancy<T, D, SHARE>())) void attn_dq_kernel(const AttnArgs a) {
    constexpr int kWaves = bwd_waves<T, D, SHARE>(), BK = bwd_rows<T, D, SHARE>(), kT = BK / 32, kD = D / 32;
    constexpr int kE = Mma<T>::kE, kK = Mma<T>::kK, kC = D / kK, kM = 32 / kK;
    constexpr int kTile = BK * D * (int)sizeof(T), kLds = SHARE == 4 ? kTile : kWaves * kTile, kSharers = SHARE == 4 ? 4 : 1;
    constexpr bool kRows = SHARE == 0;
    __shared__ __align__(16) char keys0[kLds], keys1[kLds], values0[kLds], values1[kLds];
    __shared__ int votes[2 * kWaves];
    extern __shared__ float tab[];   // the bias by distance, sums by distance - two arrays of that size for each wavefront -, the buckets
    const int wave = uniform(threadIdx.x >> 6), lane = lane_id(), col = lane & 31, half = lane >> 5;
    const uint32_t per_head = SHARE == 4 ? (uint32_t)a.V : ((uint32_t)a.V + kWaves - 1) / kWaves;
    const uint32_t groups = per_head * (uint32_t)a.H, wg = die_order(groups);
    if (wg >= groups) return;
    int head;
    uint32_t item;
    head_and_item<SHARE>(wg, per_head, a.H, head, item);
    const int size = tab_size(a.far);
    const uint32_t v = SHARE == 4 ? item : item * kWaves + wave;
    uint16_t* const bucket = reinterpret_cast<uint16_t*>(tab + size * (1 + 2 * kWaves));
    if (BIAS) {
        fill_bias(tab, a, head, 1, 64 * kWaves, bucket);
        for (int n = threadIdx.x; n < 2 * kWaves * size; n += 64 * kWaves) tab[size + n] = 0.f;
        __syncthreads();
    }
    if (v >= (uint32_t)a.V) return;
    float* const part = BIAS ? a.part_bias + ((int64_t)head * a.V + v) * a.buckets : nullptr;
    const int me = SHARE == 4 ? threadIdx.x : lane, of = SHARE == 4 ? 64 * kWaves : 64;   // of the unit's lanes
    const bool looks = !kRows && head == 0 && (SHARE == 1 || wave == 0) && v < (uint32_t)a.N;
    const int64_t peek = looks ? sequence_numbers(a, v) : 0;
    Sequence q;
    int iw, first, pos, wave_last, tiles, jbase = 0, lo = 0, end = 0;
    int own_lo = 0, own_end = 0, own_pos = 0;   // SHARE = 0: this column's own keys, and its place among all rows of k
    int back, on;                               // the furthest that a key lies behind and ahead of a query here
    bool is;
    int64_t row;
    if constexpr (kRows) {
        if (head == 0) judge_all(a, v, a.V);
        q.q0 = (int64_t)v * 32;
        q.k0 = 0;
        q.nk = (int)a.k_rows;
        q.nq = 32;
        const LaneSequence mine = lane_numbers(a, lane_sequence(a.q_off, a.N, q.q0, a.q_rows));
        row = q.q0 + col;
        is = mine.fits && row >= mine.q0 && row < mine.q1;
        own_pos = (int)(mine.k1 - mine.q1 + row);
        own_lo = is ? (int)mine.k0 : 0;
        own_end = is ? (int)mine.k1 : 0;
        if (a.causal && own_pos + 1 < own_end) own_end = own_pos + 1;
        if (own_end < own_lo) own_end = own_lo;
        const bool sees = own_lo < own_end;
        back = wave_max_i32(sees ? own_pos - own_lo : -0x40000000);
        on = wave_max_i32(sees ? own_end - 1 - own_pos : -0x40000000);
        row = is ? row : 0;
        iw = first = pos = wave_last = tiles = 0;
    } else {
        const int s = find_sequence(a.q_off, a.N, v, a.block);
        const bool fits = take_sequence(a, s, sequence_numbers(a, s), q);
        const uint32_t start = (uint32_t)q.q0 / a.block + s, blocks = ((uint32_t)q.nq + a.block - 1) / a.block;
        if (!fits || v < start || v - start >= blocks) {
            if (BIAS)
                for (int b = me; b < a.buckets; b += of) part[b] = 0.f;
            return judge(a, looks, v, peek);
        }
        const int i0 = uniform((int)(blocks - 1 - (v - start)) * a.block), i = i0 + (SHARE == 4 ? wave * 32 : 0) + col;
        iw = i0 + (SHARE == 4 ? wave * 32 : 0);
        is = i < q.nq;
        first = q.nk - q.nq + iw;
        pos = first + col;
        wave_last = first + 31;
        row = q.q0 + (is ? i : 0);
        int jend = q.nk;
        if (a.causal) {
            const int last = q.nk - q.nq + (i0 + a.block < q.nq ? i0 + a.block : q.nq);
            jend = jend < last ? jend : last;
        }
        tiles = uniform(jend > 0 ? (jend + BK - 1) / BK : 0);
        back = q.nk - q.nq + i0 + a.block - 1;
        on = q.nk - 1 - (q.nk - q.nq + i0);
    }

    uint4 fq[kC], fy[kC];
    column_row<T, D>(fq, a.q.at(row, head), is, half, a.dim);
    column_row<T, D>(fy, a.dout.at(row, head), is, half, a.dim);
    if (a.negative) flip_signs<T, kC>(fq);
    float lse = a.lse[(int64_t)head * a.q_rows + row];
    // (columns without a query, rows that saw nothing: all their probabilities are 2^-inf)
    lse = !is || lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e;

    // D of a row from its few keys' P and dP, or else from the forward's result.  That was rounded, which against the sum over few keys is
    // as much as the rounding of dS and of the gradient: 4096 bfloat16 sequences of 12 events on average have dq 1.6 times as far from
    // 64 bits as a single rounding with the latter alone, 1.4 times with the former up to kFew tiles.
    constexpr int kFew = 4;
    float delta = 0.f, dsum;
    bool one, sums_only;   // all keys in one tile of 32; a first run over the keys for D alone
    // Where a row is wide, the unit's rows find their maxima and the sums below them again, in a run over the keys of its own: lse becomes the
    // maximum, weight one over the sum.
    const bool any_wide = any_sharer<SHARE>(wide_row<T>(lse), votes, wave);
    float weight = 1.f;
    const int kvh = head / a.group;
    const char* const kb = a.k.at(q.k0, kvh);
    const char* const vb = a.v.at(q.k0, kvh);
    const int own = SHARE == 4 ? 0 : wave * kTile, fw = SHARE == 4 ? wave : 0;
    auto fetch = [&](const int t, char* const kt, char* const vt, const int l) __attribute__((always_inline)) {
        Tile<T, D>::template fetch<BK, kSharers>(kt + own, kb, a.k.row, jbase + t * BK, q.nk, a.dim, fw, l);
        Tile<T, D>::template fetch<BK, kSharers>(vt + own, vb, a.v.row, jbase + t * BK, q.nk, a.dim, fw, l);
    };
    f32x16_t dq[kD];
#pragma unroll
    for (int d = 0; d < kD; ++d) dq[d] = f32x16_t{};
    float beyond = 0.f, ahead = 0.f, sum_beyond = 0.f, sum_ahead = 0.f, carry = 0.f;
    int carry_at = -1;   // the first key of the tile whose store the carry waits for
    float* const sums = tab + size * (1 + 2 * (BIAS ? wave : 0));
    if (BIAS) {
        beyond = tab[kTabMargin];
        ahead = a.causal ? 0.f : tab[2 * a.far + kTabMargin];
    }
    // dbias: what 32 keys from j0 on add to the sums by distance
    auto count = [&](const f32x16_t& g, const int j0, const int col, const int half) __attribute__((always_inline)) {
        const bool all_beyond = first - (j0 + 31) >= a.far, all_ahead = wave_last - j0 <= -a.far;
        if (all_beyond || all_ahead) {
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += g[r];
            if (all_beyond) sum_beyond += sum;
            else sum_ahead += sum;
        } else {
            // What a tile has of one distance lies on a diagonal; see diagonal_sums.  A distance of a half's array is met by two
            // neighbouring tiles and stored once, with the second.
            const float2 now = diagonal_sums(g);
            float* const to = sums + half * size + j0 - first + a.far + kTabMargin + 4 * half - col;
            *to = now.x + carry + (kRows ? *to : 0.f);   // (other columns' places may have met these distances before)
            carry = now.y;
            carry_at = j0 + 32;
        }
    };
    auto step = [&](const int t, const char* const kt_, const char* const vt_, char* const kn, char* const vn) __attribute__((always_inline)) {
        loads_done();
        if (SHARE == 4) __syncthreads();
        if (t + 1 < tiles) fetch(t + 1, kn, vn, lane);
        const char* const kt = kt_ + own;
        const char* const vt = vt_ + own;
#pragma unroll
        for (int k = 0; k < kT; ++k) {
            const int j0 = jbase + t * BK + 32 * k;
            if (!kRows && (j0 >= q.nk || (a.causal && j0 > wave_last) || iw >= q.nq)) return;
            f32x16_t x = f32x16_t{}, g = f32x16_t{};
#pragma unroll
            for (int c = 0; c < kC; ++c) x = Mma<T>::mma(Tile<T, D>::along(kt, 32 * k + col, c, half), fq[c], x);
#pragma unroll
            for (int c = 0; c < kC; ++c) g = Mma<T>::mma(Tile<T, D>::along(vt, 32 * k + col, c, half), fy[c], g);
            reads_ahead<2 * kC, 1, Mma<T>::kMfmas, 4>();
            settle<T>();
            const bool all_beyond = first - (j0 + 31) >= a.far, all_ahead = wave_last - j0 <= -a.far;
            const int at = j0 + 4 * half - pos + a.far + kTabMargin;   // of this lane's first key among the distances
            if (!BIAS) {
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale2, -lse));
            } else if (all_beyond || all_ahead) {
                const float b = (all_beyond ? beyond : ahead) - lse;
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale2, b));
            } else {
                const float* const from = tab + at;
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale2, from[8 * (r / 4) + r % 4]) - lse);
            }
            if constexpr (kRows) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((uint32_t)(j0 + 8 * (r / 4) + 4 * half + r % 4 - lo) >= (uint32_t)(end - lo)) x[r] = g[r] = 0.f;
            } else if (j0 + 32 > q.nk || (a.causal && j0 + 31 > first)) {
                const int end = a.causal && pos + 1 < q.nk ? pos + 1 : q.nk;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (j0 + 8 * (r / 4) + 4 * half + r % 4 >= end) x[r] = g[r] = 0.f;
            }
            if (sums_only || one) {
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) sum = fmaf(x[r], g[r], sum);
                dsum += sum;
                if (sums_only) continue;
                const float d = pair_sum<32>(dsum);
                delta = !kRows || lo < end ? d : delta;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) g[r] = x[r] * (g[r] - delta);
            if (BIAS) count(g, j0, col, half);
#pragma unroll
            for (int c = 0; c < kM; ++c) {
                const uint4 p = Mma<T>::pack(g, c);
#pragma unroll
                for (int d = 0; d < kD; ++d) dq[d] = Mma<T>::mma(Tile<T, D>::down(kt, 32 * k, c, d), p, dq[d]);
            }
            reads_ahead<kM * kD, Mma<T>::kDown, Mma<T>::kMfmas, 4>();
            settle<T>();
        }
    };
    // The rare ways, one tile at a time.  Their addresses and places are computed anew, so that they take no registers in the loop above.
    auto alone = [&](const int t, const int l, const auto run) __attribute__((always_inline)) {   // `run` on 32 rows of tile t after the others
        if (SHARE == 4) __syncthreads();
        fetch(t, keys0, values0, l);
        loads_done();
        if (SHARE == 4) __syncthreads();
#pragma unroll 1
        for (int k = 0; k < kT; ++k) {
            const int j0 = jbase + t * BK + 32 * k;
            if (!kRows && (j0 >= q.nk || (a.causal && j0 > wave_last) || iw >= q.nq)) return;
            run(k, j0);
        }
    };
    // the exponents of 32 keys' probabilities: their products, scaled, with their bias, less `by`
    auto exponents = [&](f32x16_t& x, const int j0, const float by, const int place, const int half) __attribute__((always_inline)) {
        const bool all_beyond = first - (j0 + 31) >= a.far, all_ahead = wave_last - j0 <= -a.far;
        if (!BIAS) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], a.scale2, -by);
        } else if (all_beyond || all_ahead) {
            const float flat = all_beyond ? beyond : ahead;
            // (a wide row's scores are rounded with their bias, as in the forward and in other tiles, and not with its difference to lse)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = any_wide ? fmaf(x[r], a.scale2, flat) - by : fmaf(x[r], a.scale2, flat - by);
        } else {
            const float* const from = tab + (j0 + 4 * half - place + a.far + kTabMargin);
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], a.scale2, from[8 * (r / 4) + r % 4]) - by;
        }
    };
    auto find_statistics = [&]() __attribute__((always_inline)) {
        const int l = anew(lane), c32 = l & 31, h = l >> 5, place = anew(pos);
        const int from = kRows ? lo : 0, to = kRows ? end : (a.causal && place + 1 < q.nk ? place + 1 : q.nk);
        float top = -__builtin_inff(), sum = 0.f, d = 0.f;
#pragma unroll 1
        for (int t = 0; t < tiles; ++t)
            alone(t, l, [&](const int k, const int j0) __attribute__((always_inline)) {
                f32x16_t x = f32x16_t{}, g = f32x16_t{};
#pragma unroll
                for (int c = 0; c < kC; ++c) x = Mma<T>::mma(Tile<T, D>::along(keys0 + own, 32 * k + c32, c, h), fq[c], x);
#pragma unroll
                for (int c = 0; c < kC; ++c) g = Mma<T>::mma(Tile<T, D>::along(values0 + own, 32 * k + c32, c, h), fy[c], g);
                settle<T>();
                exponents(x, j0, 0.f, place, h);
                float most = top;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int j = j0 + 8 * (r / 4) + 4 * h + r % 4;
                    const bool sees = j >= from && j < to;
                    x[r] = sees ? x[r] : -__builtin_inff();
                    g[r] = sees ? g[r] : 0.f;
                    most = fmaxf(most, x[r]);
                }
                most = halves_max(most);
                const float at = most == -__builtin_inff() ? 0.f : most, shrink = __builtin_amdgcn_exp2f(top - at);
                sum *= shrink;
                d *= shrink;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float p = __builtin_amdgcn_exp2f(x[r] - at);
                    sum += p;
                    d = fmaf(p, g[r], d);
                }
                top = most;
            });
        sum = pair_sum<32>(sum);
        d = pair_sum<32>(d);
        const bool found = sum != 0.f, apart = wide_row<T>(top);   // (attn_dkv_kernel goes by lse)
        lse = !found ? lse : (apart ? top : top + __builtin_amdgcn_logf(sum));
        weight = found && apart ? 1.f / sum : weight;
        delta = found ? d / sum : delta;
    };
    // The step's dS, bit by bit.  What is hidden has dS = 0, but 0 times a key that is not finite is not 0: its elements are multiplied one by one, for
    // the columns that see them (see Tile::cleaned).
    auto careful_step = [&](const int t, const bool counts) __attribute__((always_inline)) {
        const int l = anew(lane), c32 = l & 31, h = l >> 5, place = anew(pos);
        const int from = kRows ? lo : 0, to = kRows ? end : (a.causal && place + 1 < q.nk ? place + 1 : q.nk);
        alone(t, l, [&](const int k, const int j0) __attribute__((always_inline)) {
            f32x16_t x = f32x16_t{}, g = f32x16_t{};
#pragma unroll
            for (int c = 0; c < kC; ++c) x = Mma<T>::mma(Tile<T, D>::along(keys0 + own, 32 * k + c32, c, h), fq[c], x);
#pragma unroll
            for (int c = 0; c < kC; ++c) g = Mma<T>::mma(Tile<T, D>::along(values0 + own, 32 * k + c32, c, h), fy[c], g);
            reads_ahead<2 * kC, 1, Mma<T>::kMfmas, 2>();
            settle<T>();
            exponents(x, j0, lse, place, h);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int j = j0 + 8 * (r / 4) + 4 * h + r % 4;
                g[r] = j >= from && j < to ? __builtin_amdgcn_exp2f(x[r]) * weight * (g[r] - delta) : 0.f;
            }
            if (BIAS && counts) count(g, j0, c32, h);
            Tile<T, D>::add_not_finite(dq, keys0 + own, 32 * k, g, from - j0, to - j0, l);
#pragma unroll
            for (int c = 0; c < kM; ++c) {
                const uint4 p = Mma<T>::pack(g, c);
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    dq[d] = Mma<T>::mma(Tile<T, D>::cleaned(Tile<T, D>::down(keys0 + own, 32 * k, c, d, l)), p, dq[d]);
                    __builtin_amdgcn_sched_barrier(0);   // (few registers rather than many loads under way)
                }
            }
            settle<T>();
        });
    };
    // SHARE = 0: columns whose places lie as their rows do go together
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
        tiles = jbase < last ? (last - jbase + BK - 1) / BK : 0;
    };
    // the last tile's share of dbias
    auto count_rest = [&]() __attribute__((always_inline)) {
        if (BIAS && carry_at >= 0) {
            float* const to = sums + half * size + carry_at - first + a.far + kTabMargin + 4 * half - col;
            *to = carry + (kRows ? *to : 0.f);
            carry = 0.f;
            carry_at = -1;
        }
    };
    for (uint64_t todo = any_wide ? 0 : (kRows ? __ballot(is) : 1); todo;) {
        if constexpr (kRows) take_some(todo);
        else todo = 0;
        one = kT == 1 && tiles == 1;
        sums_only = tiles <= kFew && !one;
        dsum = 0.f;
        if (tiles > kFew) {
            uint4 fo[kC];
            column_row<T, D>(fo, a.o.at(row, head), is, half, a.dim);
            float d = 0.f;
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                float x[kE], y[kE];
                Frag<T>::unpack(fo[c], x);
                Frag<T>::unpack(fy[c], y);
#pragma unroll
                for (int e = 0; e < kE; ++e) d = fmaf(x[e], y[e], d);
            }
            d = pair_sum<32>(d);
            delta = !kRows || lo < end ? d : delta;
        }
        for (;;) {
            if (tiles > 0) fetch(0, keys0, values0, lane);
            for (int t = 0; t < tiles; t += 2) {
                step(t, keys0, values0, keys1, values1);
                if (t + 1 < tiles) step(t + 1, keys1, values1, keys0, values0);
            }
            if (!sums_only) break;
            sums_only = false;
            const float d = pair_sum<32>(dsum);
            delta = !kRows || lo < end ? d : delta;
            if (SHARE == 4) __syncthreads();   // (the first tile's place may still be read)
        }
        count_rest();
    }
    if (!kRows) judge(a, looks, v, peek);
    bool carefully = any_wide;
    if ((kRows || a.causal) && !any_wide) carefully = any_sharer<SHARE>(is && not_finite(dq), votes + kWaves, wave);   // (where some keys are hidden)
    if (carefully) {
#pragma unroll
        for (int d = 0; d < kD; ++d) dq[d] = f32x16_t{};
        for (uint64_t todo = kRows ? __ballot(is) : 1; todo;) {
            if constexpr (kRows) take_some(todo);
            else todo = 0;
            if (any_wide) find_statistics();
#pragma unroll 1
            for (int t = 0; t < tiles; ++t) careful_step(t, any_wide);   // (dbias has been counted otherwise)
            count_rest();
        }
    }
    if (is && half == 0) {   // for attn_dkv_kernel
        a.delta[(int64_t)head * a.q_rows + row] = delta;
        a.lse2[(int64_t)head * a.q_rows + row] = lse;
        a.weight[(int64_t)head * a.q_rows + row] = weight;
    }
    if (is) store_column<T, D>(const_cast<char*>(a.dq.at(row, head)), dq, a.scale, half, a.dim);
    if (!BIAS) return;
    // the distances that this unit has met
    const int reach = a.far + kTabMargin;
    int from = reach - (back < reach ? back : reach), to = reach + (a.causal || on < 0 ? 0 : (on < reach ? on : reach)) + 1;
    from = from < 0 ? 0 : (from > size ? size : from);
    to = to > size ? size : to;
    sum_beyond = group_sum(sum_beyond, 64);
    sum_ahead = group_sum(sum_ahead, 64);
    if (SHARE == 4) {
        __syncthreads();
        if (lane == 0) {   // the bias itself is not needed any more
            tab[2 * wave] = sum_beyond;
            tab[2 * wave + 1] = sum_ahead;
        }
        for (int t = from + (int)threadIdx.x; t < to; t += 64 * kWaves) {
            float x = 0.f;
#pragma unroll
            for (int w = 0; w < 2 * kWaves; ++w) x += tab[size * (1 + w) + t];
            tab[size + t] = x;
        }
        __syncthreads();
        sum_beyond = tab[0] + tab[2] + tab[4] + tab[6];
        sum_ahead = tab[1] + tab[3] + tab[5] + tab[7];
    } else {
        for (int t = from + lane; t < to; t += 64) sums[t] += sums[size + t];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    bucket_sums(a, part, SHARE == 4 ? tab + size : sums, bucket, from, to, sum_beyond, sum_ahead, me, of);
}

// Sums the units' shares of dbias, in their order: 8 buckets of a head a workgroup, 32 slices of the units beside each other.
__global__ __launch_bounds__(256) void attn_dbias_kernel(const AttnArgs a, void* dbias) {
    __shared__ float part[32][9];
    const int c = threadIdx.x % 8, k = threadIdx.x / 8, b = blockIdx.x * 8 + c, head = blockIdx.y;
    part[k][c] = b < a.buckets ? strided_sum(a.part_bias + (int64_t)head * a.V * a.buckets + b, a.buckets, k, a.V, 32) : 0.f;
    __syncthreads();
    if (k == 0 && b < a.buckets) {
        float t = 0.f;
        for (int i = 0; i < 32; ++i) t += part[i][c];
        param_store(dbias, a.bias_io, (int64_t)head * a.buckets + b, t);
    }
}

// A unit: `block` keys of a sequence and a key head, hp of the heads that read it one after the other.  Where a group is cut into several
// such parts, each leaves fp32 sums (part_o: [2][parts][k_rows][kv][D]), which attn_dkv_join_kernel adds up.
template <typename T, int D, int SHARE, bool BIAS>
__global__ __launch_bounds__((64 * bwd_waves<T, D, SHARE>()), (dkv_occupancy<T, D>())) void attn_dkv_kernel(const AttnArgs a) {
    constexpr int kWaves = bwd_waves<T, D, SHARE>(), BQ = bwd_rows<T, D, SHARE>(), kT = BQ / 32, kD = D / 32;
    constexpr int kK = Mma<T>::kK, kC = D / kK, kM = 32 / kK;
    constexpr int kTile = BQ * D * (int)sizeof(T), kSets = SHARE == 4 ? 1 : kWaves, kLds = kSets * kTile, kSharers = SHARE == 4 ? 4 : 1;
    constexpr bool kRows = SHARE == 0;
    __shared__ __align__(16) char rows0[kLds], rows1[kLds], grads0[kLds], grads1[kLds];
    __shared__ __align__(16) float stats0[kSets * 128], stats1[kSets * 128];   // lse and delta of 64 rows
    __shared__ int votes[kWaves];
    extern __shared__ float tab[];
    const int wave = uniform(threadIdx.x >> 6), lane = lane_id(), col = lane & 31, half = lane >> 5;
    const int parts = a.splits, hp = a.pack;
    const uint32_t per_head = SHARE == 4 ? (uint32_t)a.V : ((uint32_t)a.V + kWaves - 1) / kWaves;
    const uint32_t groups = per_head * (uint32_t)(a.kv * parts), wg = die_order(groups);
    if (wg >= groups) return;
    int hh;
    uint32_t item;
    head_and_item<SHARE>(wg, per_head, a.kv * parts, hh, item);
    const int kvh = hh / parts, part = hh - kvh * parts, head0 = kvh * a.group + part * hp, size = tab_size(a.far);
    const uint32_t v = SHARE == 4 ? item : item * kWaves + wave;
    if (BIAS && SHARE != 4) {
        fill_bias(tab, a, head0, hp, 64 * kWaves);
        __syncthreads();
    }
    if (v >= (uint32_t)a.V) return;
    Sequence q;
    int j0, jw, j, lead, t0 = 0, tiles, ibase = 0, lo = 0, end = 0;
    int own_lo = 0, own_end = 0, own_lead = 0;   // SHARE = 0: the rows of q that see this column's key, and how far their places lie from their rows
    bool is, writes;
    if constexpr (kRows) {
        if (hh == 0) judge_all(a, v, a.V);
        q.k0 = (int64_t)v * 32;
        q.q0 = 0;
        q.nq = (int)a.q_rows;
        q.nk = q.cap = 32;
        const LaneSequence mine = lane_numbers(a, lane_sequence(a.k_off, a.N, q.k0, a.k_rows));
        const int64_t row = q.k0 + col;
        is = writes = mine.fits && row >= mine.k0 && row < mine.k1;
        own_lead = (int)(mine.k1 - mine.q1);
        own_lo = is ? (int)mine.q0 : 0;
        own_end = is ? (int)mine.q1 : 0;
        if (is && a.causal && (int)row - own_lead > own_lo) own_lo = (int)row - own_lead;
        if (own_end < own_lo) own_end = own_lo;
        j0 = jw = 0;
        j = col;
        lead = tiles = 0;
        if (!__any(is)) return;
    } else {
        const int s = find_sequence(a.k_off, a.N, v, a.block);
        if (!take_sequence(a, s, sequence_numbers(a, s), q)) return;
        const uint32_t start = (uint32_t)q.k0 / a.block + s, blocks = ((uint32_t)q.cap + a.block - 1) / a.block;
        if (v < start || v - start >= blocks) return;
        j0 = uniform((int)(v - start) * a.block);
        jw = j0 + (SHARE == 4 ? wave * 32 : 0);
        j = jw + col;
        is = j < q.nk;
        writes = j < q.cap;
        // the queries that see these keys: all, or from the one in the first key's place on
        lead = q.nk - q.nq;   // the first query's place
        if (a.causal && j0 > lead) t0 = (j0 - lead) / BQ;
        const int all = j0 < q.nk ? (q.nq + BQ - 1) / BQ : 0;
        t0 = uniform(t0 < all ? t0 : all);
        tiles = uniform(all - t0);
    }

    uint4 fk[kC], fv[kC];
    column_row<T, D>(fk, a.k.at(q.k0 + (is ? j : 0), kvh), is, half, a.dim);
    column_row<T, D>(fv, a.v.at(q.k0 + (is ? j : 0), kvh), is, half, a.dim);
    if (a.negative) flip_signs<T, kC>(fk);

    const int own = SHARE == 4 ? 0 : wave * kTile, own_stats = SHARE == 4 ? 0 : wave * 128, fw = SHARE == 4 ? wave : 0;
    auto fetch = [&](const int g, const int t, char* const qt, char* const yt, float* const st, const int l_) __attribute__((always_inline)) {
        const int head = head0 + g;
        Tile<T, D>::template fetch<BQ, kSharers>(qt + own, a.q.at(q.q0, head), a.q.row, ibase + t * BQ, q.nq, a.dim, fw, l_);
        Tile<T, D>::template fetch<BQ, kSharers>(yt + own, a.dout.at(q.q0, head), a.dout.row, ibase + t * BQ, q.nq, a.dim, fw, l_);
        if (SHARE != 4 || wave < 2) {
            const int i = ibase + t * BQ + l_;
            const bool there = l_ < BQ && i < q.nq;
            const int64_t at = (int64_t)head * a.q_rows + q.q0 + i;
            const float* const l = there ? a.lse2 + at : &attn_inf;
            const float* const d = there ? a.delta + at : reinterpret_cast<const float*>(&attn_zeros);
            if (SHARE != 4 || wave == 0)
                load_lds<4>(l, st + own_stats);
            if (SHARE != 4 || wave == 1)
                load_lds<4>(d, st + own_stats + 64);
        }
    };
    f32x16_t dk[kD], dv[kD];
#pragma unroll
    for (int d = 0; d < kD; ++d) dk[d] = dv[d] = f32x16_t{};
    bool met_wide = false;   // (wide rows' probabilities have weights: see below)
    // the step after (g, t) is (g, t + 1) or the next head's first
    auto step = [&](const int g, const int t, const bool more, const char* const qt_, const char* const yt_, const float* const st_, char* const qn,
                    char* const yn, float* const sn) __attribute__((always_inline)) {
        loads_done();
        if (SHARE == 4) __syncthreads();
        if (more) {
            const bool next = t + 1 == t0 + tiles;
            fetch(next ? g + 1 : g, next ? t0 : t + 1, qn, yn, sn, lane);
        }
        if (BIAS && SHARE == 4 && t == t0) {
            fill_bias(tab, a, head0 + g, 1, 64 * kWaves);
            __syncthreads();
        }
        const char* const qt = qt_ + own;
        const char* const yt = yt_ + own;
        const float* const ht = SHARE == 4 ? tab : tab + g * size;
        met_wide |= wide_row<T>(st_[own_stats + lane % BQ]);
#pragma unroll
        for (int k = 0; k < kT; ++k) {
            const int i0 = ibase + t * BQ + 32 * k, first = lead + i0;   // the first query and its place
            if (!kRows && (i0 >= q.nq || jw >= q.nk)) return;
            if (!kRows && a.causal && first + 31 < jw) continue;
            f32x16_t x = f32x16_t{}, g_ = f32x16_t{};
#pragma unroll
            for (int c = 0; c < kC; ++c) x = Mma<T>::mma(Tile<T, D>::along(qt, 32 * k + col, c, half), fk[c], x);
#pragma unroll
            for (int c = 0; c < kC; ++c) g_ = Mma<T>::mma(Tile<T, D>::along(yt, 32 * k + col, c, half), fv[c], g_);
            reads_ahead<2 * kC, 1, Mma<T>::kMfmas, 4>();
            settle<T>();
            const float* const lse = st_ + own_stats + 32 * k + 4 * half;
            const bool all_beyond = first - (jw + 31) >= a.far, all_ahead = first + 31 - jw <= -a.far;
            if (BIAS && (all_beyond || all_ahead)) {
                const float flat = all_beyond ? ht[kTabMargin] : (a.causal ? 0.f : ht[2 * a.far + kTabMargin]);
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], a.scale2, flat);
            } else if (BIAS) {
                const float* const from = ht + (j - first - 4 * half + a.far + kTabMargin) - 27;
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = fmaf(x[r], a.scale2, from[27 - 8 * (r / 4) - r % 4]);
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float4 l4 = *reinterpret_cast<const float4*>(lse + 8 * n), d4 = *reinterpret_cast<const float4*>(lse + 64 + 8 * n);
                const float l[4] = {l4.x, l4.y, l4.z, l4.w}, d[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * n + e;
                    if (!BIAS) x[r] = __builtin_amdgcn_exp2f(fmaf(x[r], a.scale2, -l[e]));
                    else x[r] = __builtin_amdgcn_exp2f(x[r] - l[e]);
                    g_[r] = x[r] * (g_[r] - d[e]);
                }
            }
            if constexpr (kRows) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((uint32_t)(i0 + 8 * (r / 4) + 4 * half + r % 4 - lo) >= (uint32_t)(end - lo)) x[r] = g_[r] = 0.f;
            } else if (a.causal && first < jw + 31) {   // hidden: queries before the key's place
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (first + 8 * (r / 4) + 4 * half + r % 4 < j) x[r] = g_[r] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < kM; ++c) {
                const uint4 p = Mma<T>::pack(x, c), ds = Mma<T>::pack(g_, c);
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    dv[d] = Mma<T>::mma(Tile<T, D>::down(yt, 32 * k, c, d), p, dv[d]);
                    dk[d] = Mma<T>::mma(Tile<T, D>::down(qt, 32 * k, c, d), ds, dk[d]);
                }
            }
            reads_ahead<2 * kM * kD, Mma<T>::kDown, Mma<T>::kMfmas, 4>();
            settle<T>();
        }
    };
    // The step with weights, and with care for elements of q and dout that are not finite, as in attn_dq_kernel; otherwise the same bit by bit.
    auto careful_step = [&](const int g, const int t) __attribute__((always_inline)) {
        const int l = anew(lane), c32 = l & 31, h = l >> 5, place = anew(j);
        if (SHARE == 4) __syncthreads();
        fetch(g, t, rows0, grads0, stats0, l);
        if (SHARE != 4 || wave == 0) {   // the rows' weights
            const int i = ibase + t * BQ + l;
            const float* const w = a.weight + (int64_t)(head0 + g) * a.q_rows + q.q0 + i;
            load_lds<4>(l < BQ && i < q.nq ? w : reinterpret_cast<const float*>(&attn_zeros), stats1 + own_stats);
        }
        if (BIAS && SHARE == 4 && t == t0) fill_bias(tab, a, head0 + g, 1, 64 * kWaves);
        loads_done();
        if (SHARE == 4) __syncthreads();
#pragma unroll 1
        for (int k = 0; k < kT; ++k) {
            const int i0 = ibase + t * BQ + 32 * k, first = lead + i0;
            if (!kRows && (i0 >= q.nq || jw >= q.nk)) return;
            if (!kRows && a.causal && first + 31 < jw) continue;
            f32x16_t x = f32x16_t{}, g_ = f32x16_t{};
#pragma unroll
            for (int c = 0; c < kC; ++c) x = Mma<T>::mma(Tile<T, D>::along(rows0 + own, 32 * k + c32, c, h), fk[c], x);
#pragma unroll
            for (int c = 0; c < kC; ++c) g_ = Mma<T>::mma(Tile<T, D>::along(grads0 + own, 32 * k + c32, c, h), fv[c], g_);
            reads_ahead<2 * kC, 1, Mma<T>::kMfmas, 2>();
            settle<T>();
            const float* const lse = stats0 + own_stats + 32 * k + 4 * h;
            const float* const ht = SHARE == 4 ? tab : tab + g * size;
            const float* const weights = stats1 + own_stats + 32 * k + 4 * h;
            const bool all_beyond = first - (jw + 31) >= a.far, all_ahead = first + 31 - jw <= -a.far;
            float flat = 0.f;
            if (BIAS && (all_beyond || all_ahead)) flat = all_beyond ? ht[kTabMargin] : (a.causal ? 0.f : ht[2 * a.far + kTabMargin]);
            const bool by_distance = BIAS && !all_beyond && !all_ahead;
            const float* const near = by_distance ? ht + (place - first - 4 * h + a.far + kTabMargin) - 27 : nullptr;
            const int from = kRows ? lo - i0 : (a.causal ? place - first : 0), to = kRows ? end - i0 : 32;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int e = 8 * (r / 4) + r % 4, i = 4 * h + e;
                if (!BIAS) x[r] = fmaf(x[r], a.scale2, -lse[e]);
                else x[r] = fmaf(x[r], a.scale2, by_distance ? near[27 - e] : flat) - lse[e];
                x[r] = __builtin_amdgcn_exp2f(x[r]);
                g_[r] = x[r] * (g_[r] - lse[64 + e]);
                const bool sees = i >= from && i < to;
                x[r] = sees ? x[r] * weights[e] : 0.f;
                g_[r] = sees ? g_[r] * weights[e] : 0.f;
                if (r % 4 == 3) __builtin_amdgcn_sched_barrier(0);   // (few registers rather than many loads under way)
            }
            Tile<T, D>::add_not_finite(dv, grads0 + own, 32 * k, x, from, to, l);
            Tile<T, D>::add_not_finite(dk, rows0 + own, 32 * k, g_, from, to, l);
#pragma unroll
            for (int c = 0; c < kM; ++c) {
                const uint4 p = Mma<T>::pack(x, c), ds = Mma<T>::pack(g_, c);
#pragma unroll
                for (int d = 0; d < kD; ++d) {
                    dv[d] = Mma<T>::mma(Tile<T, D>::cleaned(Tile<T, D>::down(grads0 + own, 32 * k, c, d, l)), p, dv[d]);
                    dk[d] = Mma<T>::mma(Tile<T, D>::cleaned(Tile<T, D>::down(rows0 + own, 32 * k, c, d, l)), ds, dk[d]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            settle<T>();
        }
    };
    // SHARE = 0: keys whose queries' places lie alike go together
    auto take_some = [&](uint64_t& todo) __attribute__((always_inline)) {
        lead = uniform(bcast_lane(own_lead, __ffsll((unsigned long long)todo) - 1)) - (int)q.k0;
        const bool mine = is && own_lead - (int)q.k0 == lead;
        todo &= ~__ballot(mine);
        lo = mine ? own_lo : 0;
        end = mine ? own_end : 0;
        ibase = wave_min_i32(lo < end ? lo : 0x7FFFFFFF);
        const int last = wave_max_i32(lo < end ? end : 0);
        tiles = ibase < last ? (last - ibase + BQ - 1) / BQ : 0;
    };
    for (uint64_t todo = kRows ? __ballot(is) : 1; todo;) {
        if constexpr (kRows) take_some(todo);
        else todo = 0;
        const int steps = tiles * hp;
        if (steps > 0) fetch(0, t0, rows0, grads0, stats0, lane);
        int g = 0, t = t0;
        for (int n = 0; n < steps; n += 2) {
            step(g, t, n + 1 < steps, rows0, grads0, stats0, rows1, grads1, stats1);
            if (++t == t0 + tiles) { t = t0; ++g; }
            if (n + 1 >= steps) break;
            step(g, t, n + 2 < steps, rows1, grads1, stats1, rows0, grads0, stats0);
            if (++t == t0 + tiles) { t = t0; ++g; }
        }
    }
    if (any_sharer<SHARE>(met_wide || ((kRows || a.causal) && is && (not_finite(dk) || not_finite(dv))), votes, wave)) {
#pragma unroll
        for (int d = 0; d < kD; ++d) dk[d] = dv[d] = f32x16_t{};
        for (uint64_t todo = kRows ? __ballot(is) : 1; todo;) {
            if constexpr (kRows) take_some(todo);
            else todo = 0;
#pragma unroll 1
            for (int g = 0; g < hp; ++g)
#pragma unroll 1
                for (int t = t0; t < t0 + tiles; ++t) careful_step(g, t);
        }
    }
    if (!writes) return;
    const float by = is ? 1.f : 0.f;   // (a cache's room: zeros)
    if (!is) {
#pragma unroll
        for (int d = 0; d < kD; ++d) dk[d] = dv[d] = f32x16_t{};
    }
    const int64_t row = q.k0 + j;
    if (parts > 1) {
        char* const to = reinterpret_cast<char*>(a.part_o + (((int64_t)part * a.k_rows + row) * a.kv + kvh) * D);
        store_column<float, D>(to, dk, by, half, D);
        store_column<float, D>(to + (int64_t)parts * a.k_rows * a.kv * D * 4, dv, by, half, D);
    } else {
        store_column<T, D>(const_cast<char*>(a.dk.at(row, kvh)), dk, a.scale, half, a.dim);
        store_column<T, D>(const_cast<char*>(a.dv.at(row, kvh)), dv, 1.f, half, a.dim);
    }
}

// Adds up the parts of a group's heads, in their order: four elements a lane, every row.  All rows are some sequence's; those of one that does
// not fit, which has been reported, get what the workspace holds.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_dkv_join_kernel(const AttnArgs a) {
    const int64_t per = (int64_t)a.kv * (D / 4), n = a.k_rows * per;
    const int64_t plane = a.k_rows * a.kv * D;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per;
        const int rest = (int)(i - row * per), kvh = rest / (D / 4), e = (rest - kvh * (D / 4)) * 4;
        if (e >= a.dim) continue;
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int p = 0; p < a.splits; ++p) {
                const float4 x = *reinterpret_cast<const float4*>(a.part_o + (which * a.splits + p) * plane + (row * a.kv + kvh) * D + e);
                sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
            }
            const float by = which == 0 ? a.scale : 1.f;
            char* const to = const_cast<char*>((which == 0 ? a.dk : a.dv).at(row, kvh));
            if constexpr (sizeof(T) == 2)
                *reinterpret_cast<uint2*>(to + 2 * e) = make_uint2(pack2((const T*)nullptr, sum.x * by, sum.y * by), pack2((const T*)nullptr, sum.z * by, sum.w * by));
            else *reinterpret_cast<float4*>(to + 4 * e) = make_float4(sum.x * by, sum.y * by, sum.z * by, sum.w * by);
        }
    }
}

// How the backward shares out its work: queries and keys of long sequences by 128, of short ones by 32; the heads of a group in
// parts where there would be too few workgroups of keys to fill the chip: 768 that share tiles, 4096 wavefronts on their own (16 sequences of
// 2500, 8 heads of 64 over 2 binary16, dk and dv and the join, us: 256 / 768 / 2048 of them 403 / 412 / 400; 4 of them 199 / 128 / 129).
// Short sequences share wavefronts where there are many (see kManyUnits); of dk and dv those of narrow heads and of 64 fp32 elements:
// wavefronts of one sequence / shared ones, 4096 sequences of 12 events on average, 4 heads of 32 bfloat16 58 / 41, 8 of 64 fp32 566 / 272;
// 1024 of 40, 33 / 27, 310 / 217.  (8 heads of 64 bfloat16, for which the shared ones are not built yet: 175 / 107, 92 / 72.)
AttnBackwardPlan attn_backward_plan(const AttnShape& sh) {
    AttnBackwardPlan p;
    const int64_t mean_q = (sh.q_rows + sh.N - 1) / sh.N, mean_k = (sh.k_rows + sh.N - 1) / sh.N;
    const int group = sh.H / sh.kv;
    p.D = sh.dim <= 32 ? 32 : (sh.dim <= 64 ? 64 : 128);
    const int64_t few = p.D == 32 ? 128 : (p.D == 64 ? (sh.narrow ? 192 : 384) : 64);
    p.shared_q = !attn_few(mean_q, mean_k, few);
    p.rows_q = !p.shared_q && !sh.caches && mean_k <= 2 * mean_q && (sh.q_rows / 32 + sh.N) * sh.H >= kManyUnits;
    p.block_q = p.shared_q ? 128 : 32;
    p.V_q = p.rows_q ? (sh.q_rows + 31) / 32 : sh.q_rows / p.block_q + sh.N;
    const int64_t tables = sh.buckets ? (int64_t)group * (2 * sh.far + 1 + 2 * kTabMargin) * 4 : 0;
    p.shared_k = tables > kTabBytes || !attn_few(mean_k, mean_q, p.D == 128 && sh.narrow ? INT64_MAX : few);
    p.rows_k = (p.D == 32 || (p.D == 64 && !sh.narrow)) && !p.shared_k && !sh.caches && mean_q <= 2 * mean_k && (sh.k_rows / 32 + sh.N) * sh.kv >= kManyUnits;
    p.block_k = p.shared_k ? 128 : 32;
    p.V_k = p.rows_k ? (sh.k_rows + 31) / 32 : sh.k_rows / p.block_k + sh.N;
    const int64_t units = (sh.k_rows / p.block_k + 1) * sh.kv, enough = p.shared_k ? 768 : 4096;
    p.parts = 1;
    while (p.parts < group && units * p.parts < enough) {
        int next = p.parts + 1;
        while (group % next != 0) ++next;
        p.parts = next;
    }
    p.delta = 3 * (((size_t)sh.H * (size_t)sh.q_rows * 4 + 255) & ~(size_t)255);   // with lse2 and weight
    p.part_bias = sh.buckets ? ((size_t)sh.H * (size_t)p.V_q * (size_t)sh.buckets * 4 + 255) & ~(size_t)255 : 0;
    p.part_kv = p.parts > 1 ? 2 * (size_t)p.parts * (size_t)sh.k_rows * (size_t)sh.kv * (size_t)p.D * 4 : 0;
    p.grid_ok = (int64_t)sh.H * p.V_q < ((int64_t)1 << 31) - 64 && (int64_t)sh.kv * p.parts * p.V_k < ((int64_t)1 << 31) - 64;
    return p;
}
size_t attn_backward_workspace(const AttnShape& sh) {   // (large tables of distances make the keys' units large)
    AttnShape any = sh;
    any.caches = true;   // (which has the most units)
    size_t most = 0;
    for (const int far : {0, kAttnMaxFar})
        for (const bool narrow : {false, true}) {
            any.far = far;
            any.narrow = narrow;
            const AttnBackwardPlan p = attn_backward_plan(any);
            most = std::max(most, p.delta + p.part_bias + p.part_kv);
        }
    return most;
}

static hipError_t room_for(const void* kernel, const size_t bytes) {
    return bytes > (32 << 10) ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : hipSuccess;
}
template <typename T, int D, int SHARE, bool BIAS>
static hipError_t launch_dq(const AttnArgs& a, hipStream_t s) {
    constexpr int kWaves = bwd_waves<T, D, SHARE>();
    const size_t table = BIAS ? (size_t)(2 * a.far + 1 + 2 * kTabMargin) * ((1 + 2 * kWaves) * 4 + 2) : 0;
    const uint64_t per_head = SHARE == 4 ? (uint64_t)a.V : ((uint64_t)a.V + kWaves - 1) / kWaves;
    const hipError_t e = room_for(reinterpret_cast<const void*>(attn_dq_kernel<T, D, SHARE, BIAS>), table);
    if (e != hipSuccess) return e;
    attn_dq_kernel<T, D, SHARE, BIAS><<<die_grid(per_head * a.H), 64 * kWaves, table, s>>>(a);
    return hipGetLastError();
}
template <typename T, int D, int SHARE, bool BIAS>
static hipError_t launch_dkv(const AttnArgs& a, hipStream_t s) {
    constexpr int kWaves = bwd_waves<T, D, SHARE>();
    const size_t table = BIAS ? (size_t)(SHARE == 4 ? 1 : a.pack) * (2 * a.far + 1 + 2 * kTabMargin) * 4 : 0;
    const uint64_t per_head = SHARE == 4 ? (uint64_t)a.V : ((uint64_t)a.V + kWaves - 1) / kWaves;
    attn_dkv_kernel<T, D, SHARE, BIAS><<<die_grid(per_head * a.kv * a.splits), 64 * kWaves, table, s>>>(a);
    return hipGetLastError();
}
template <typename T, int D>
static hipError_t launch_dim(const tbe_handle* h, AttnArgs a, const AttnBackwardPlan& p, void* dbias, hipStream_t s) {
    hipError_t e = hipSuccess;
    if (a.q_rows > 0) {
        a.V = (int)p.V_q; a.block = p.block_q;
        LaunchTimer tm(h, s, "attention_dq");
        if (p.shared_q) e = a.bias ? launch_dq<T, D, 4, true>(a, s) : launch_dq<T, D, 4, false>(a, s);
        else if (p.rows_q) e = a.bias ? launch_dq<T, D, 0, true>(a, s) : launch_dq<T, D, 0, false>(a, s);
        else e = a.bias ? launch_dq<T, D, 1, true>(a, s) : launch_dq<T, D, 1, false>(a, s);
        tm.done();
        if (e != hipSuccess) return e;
    }
    if (dbias) {
        a.V = a.q_rows > 0 ? (int)p.V_q : 0;
        LaunchTimer tm(h, s, "attention_dbias");
        attn_dbias_kernel<<<dim3((a.buckets + 7) / 8, a.H), 256, 0, s>>>(a, dbias);
        tm.done();
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.k_rows == 0) return e;
    a.V = (int)p.V_k; a.block = p.block_k; a.splits = p.parts; a.pack = a.group / p.parts;
    {
        LaunchTimer tm(h, s, "attention_dkv");
        const auto shared = [&] {
            if constexpr (sizeof(T) == 2 && D == 128) return launch_dkv<T, D, 4, true>(a, s);   // (for large tables only)
            else return a.bias ? launch_dkv<T, D, 4, true>(a, s) : launch_dkv<T, D, 4, false>(a, s);
        };
        const auto rows = [&] {
            if constexpr (D == 32 || (D == 64 && sizeof(T) == 4)) return a.bias ? launch_dkv<T, D, 0, true>(a, s) : launch_dkv<T, D, 0, false>(a, s);
            else return hipErrorInvalidValue;   // (not planned)
        };
        if (p.shared_k) e = shared();
        else if (p.rows_k) e = rows();
        else e = a.bias ? launch_dkv<T, D, 1, true>(a, s) : launch_dkv<T, D, 1, false>(a, s);
        tm.done();
    }
    if (e != hipSuccess || p.parts == 1) return e;
    LaunchTimer tm(h, s, "attention_dkv_join");
    const int64_t lanes = a.k_rows * a.kv * (D / 4), want = (lanes + 255) / 256;
    attn_dkv_join_kernel<T, D><<<(unsigned)(want < 8192 ? want : 8192), 256, 0, s>>>(a);
    tm.done();
    return hipGetLastError();
}
template <typename T>
static hipError_t launch_type(const tbe_handle* h, const AttnArgs& a, const AttnBackwardPlan& p, void* dbias, hipStream_t s) {
    return p.D == 32 ? launch_dim<T, 32>(h, a, p, dbias, s) : (p.D == 64 ? launch_dim<T, 64>(h, a, p, dbias, s) : launch_dim<T, 128>(h, a, p, dbias, s));
}

hipError_t launch_attention_backward(const tbe_handle* h, AttnArgs a, const AttnBackwardPlan& p, int io, void* dbias, void* workspace, hipStream_t s) {
    char* const ws = static_cast<char*>(workspace);
    a.delta = reinterpret_cast<float*>(ws);
    a.lse2 = reinterpret_cast<float*>(ws + p.delta / 3);
    a.weight = reinterpret_cast<float*>(ws + p.delta / 3 * 2);
    a.part_bias = reinterpret_cast<float*>(ws + p.delta);
    a.part_o = reinterpret_cast<float*>(ws + p.delta + p.part_bias);
    return io == 0 ? launch_type<float>(h, a, p, dbias, s) : (io == 1 ? launch_type<__half>(h, a, p, dbias, s) : launch_type<bf16_t>(h, a, p, dbias, s));
}

}  // namespace tbe
