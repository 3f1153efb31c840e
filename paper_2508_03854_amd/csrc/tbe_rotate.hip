// Heads of queries and keys, normed and rotated by their rows' positions, and the gradients.
//   forward   z = x w / sqrt(1/n sum x^2 + eps)  (or z = x);   y = z with every pair (z_a, z_b) of the first `turned` elements turned:
//             y_a = A (z_a cos t - z_b sin t),  y_b = A (z_b cos t + z_a sin t),  t = position * frequency of the pair
//   backward  g: dy turned back (by -t, times A);  dx = g, or with r = 1 / sqrt(1/n sum x^2 + eps), h = x r, u = g w:
//             dx = r (u - h 1/n sum u h),  dw = sum over rows and heads of g h
// Bound: the stream, every element read once and written once.  A head's elements stay in registers between its sum and its turn; a pair lies
// in one lane, in either layout, so that nothing but the sum crosses lanes.  The turns are counted in 64 bits and reduced to an eighth of a turn
// before they become fp32; a wavefront finds sine and cosine of its rows' pairs together, once for the heads that it has (every lane for its own pairs:
// 322 us where this takes 288, gradients 365 / 268).  Measured: 131,071 rows of 16 and 4 heads of 128, bfloat16, normed: 270 us, 5.0 TB/s; gradients of 65,537 of
// them, the weights' among them: 204 and 9 us; 60,001 rows of 16 heads of 80 fp32, 32 elements turned in neighbouring pairs: 137; 40,003 of 24 heads of 64
// binary16, 24 turned, gradients: 55, 4.5 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "tbe_elems.h"
#include "tbe_internal.h"

namespace tbe {

// Cosine and sine of a number of turns.  What is left after whole and quarter turns are taken off, at most an eighth of a turn, is rounded to
// fp32 once (by at most 2^-24 of its value); the series end where the next term is below 2^-28 (sine) and 2^-32 (cosine).
__device__ __forceinline__ float2 cos_sin(double turns) {
    turns -= __builtin_rint(turns);
    const float quarters = rintf(4.f * (float)turns);
    const float t = (float)(fma(-0.25, (double)quarters, turns) * 6.283185307179586477);
    const float q = t * t;
    float s = fmaf(q, 1.f / 362880.f, -1.f / 5040.f);
    s = fmaf(q, s, 1.f / 120.f);
    s = fmaf(q, s, -1.f / 6.f);
    s = fmaf(q * t, s, t);
    float c = fmaf(q, -1.f / 3628800.f, 1.f / 40320.f);
    c = fmaf(q, c, -1.f / 720.f);
    c = fmaf(q, c, 1.f / 24.f);
    c = fmaf(q, c, -0.5f);
    c = fmaf(q, c, 1.f);
    const int k = (int)quarters;
    const float a = k & 1 ? s : c, b = k & 1 ? c : s;
    return make_float2(k & 2 ? (k & 1 ? a : -a) : (k & 1 ? -a : a), k & 2 ? -b : b);
}

// The n elements at p as they are; those behind them are 0 and are not read.
template <typename T>
__device__ __forceinline__ uint4 load_some(const T* p, const int n) {
    constexpr int kN = Frag<T>::kN;
    if (n == kN) return Frag<T>::load(p);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < kN; ++i)
        if (i < n) {
            if constexpr (kN == 4) w[i] = __float_as_uint(p[i]);
            else w[i / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(p)[i] << (16 * (i % 2));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, const int n, const float (&x)[Frag<T>::kN]) {
    constexpr int kN = Frag<T>::kN;
    if (n == kN) {
        Frag<T>::store(p, x);
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (i < n) p[i] = elem_round<T>(x[i]);
    }
}
// A run of `from` .. that holds less than kN elements is moved back to kN of them, if there are so many from `lo` on (and, where pairs follow
// each other, at an even distance): a lane then has some that its neighbour has too, the first `again` of its run.  Both make the same of them; sums
// leave them out here.  (One by one they took 170 us where this takes 91: 40,003 rows of 24 heads of 64 binary16, 24 elements turned.)
__device__ __forceinline__ void move_back(int& from, int& n, int& again, const int lo, const int kN, const bool even) {
    again = 0;
    if (n > 0 && n < kN && from + n - kN >= lo && !(even && ((kN - n) & 1))) {
        again = kN - n;
        from -= again;
        n = kN;
    }
}

// Below this eps the squares of small heads count, however far below fp32's smallest numbers they lie, and the kernels that take heads of any size run.
// Among the others (eps is more than all that fp32 loses of such squares) a branch in the heads' loop costs too much: 131,071 rows of 20 heads of 128
// bfloat16 271 us without / 281 with it, gradients of 65,537 of them 216 / 220, of 60,000 rows of 12 heads of 96, 72 elements turned, 141 / 155.
constexpr float kEpsAny = 0x1p-100f;

// 1 / sqrt(1/n sum x^2 + eps) of a head that a group of lanes has, each the two runs a and b.  ANY: where the mean of the squares, eps included, leaves
// fp32's range or comes near its lower end, it is that of the head times a power of two, `by` (otherwise 1), with which the largest magnitude, or
// eps's root if that is larger, lies next to 1.  All lanes of a wavefront together.
template <bool ANY, int kN>
__device__ __forceinline__ float head_rstd(const float (&a)[kN], const float (&b)[kN], const int again_a, const int again_b, const int lanes, const float inv,
                                           const float eps, const bool here, float& by) {
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < kN; ++j) q = j < again_a ? q : fmaf(a[j], a[j], q);
#pragma unroll
    for (int j = 0; j < kN; ++j) q = j < again_b ? q : fmaf(b[j], b[j], q);
    float m = group_sum(q, lanes) * inv + eps;
    by = 1.f;
    if constexpr (!ANY) return 1.f / sqrtf(m);
    const bool beyond = here && !(m >= kEpsAny && m < __builtin_inff());   // (NaN too)
    if (__any(beyond)) {
        uint32_t top = __float_as_uint(sqrtf(eps));
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            top = max(top, __float_as_uint(a[j]) & 0x7FFFFFFFu);
            top = max(top, __float_as_uint(b[j]) & 0x7FFFFFFFu);
        }
        for (int w = 1; w < lanes; w <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, w));
        int e = (int)(top >> 23) - 127;
        e = e < -126 ? -126 : (e > 126 ? 126 : e);
        by = beyond ? __uint_as_float((uint32_t)(127 - e) << 23) : 1.f;
        q = 0.f;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const float x = a[j] * by, y = b[j] * by;
            q = j < again_a ? q : fmaf(x, x, q);
            q = j < again_b ? q : fmaf(y, y, q);
        }
        q = group_sum(q, lanes) * inv + eps * by * by;   // (eps times `by` twice is at most 4)
        m = beyond ? q : m;
    }
    return 1.f / sqrtf(m);
}

__device__ __forceinline__ void turn(const bool turned, const float2 cs, float& x, float& y) {
    const float a = x, b = y;
    x = turned ? a * cs.x - b * cs.y : a;
    y = turned ? b * cs.x + a * cs.y : b;
}

// q or k.  Wavefronts take units: `per` rows, of each `beside` heads beside each other, `turns` times; `pieces` units cover all heads of the rows.
struct TurnPart {
    const void *x, *dy, *weight;
    void* y;
    int64_t x_row, x_head, dy_row, dy_head, y_row, y_head;   // elements
    float* partial;   // [blocks][dim], or null
    uint32_t units, blocks;
    int heads, beside, per, turns, pieces;
};
struct TurnArgs {
    TurnPart part[2];
    IdxView positions;
    const double* frequencies;
    int64_t rows;
    int dim, half, lanes, param_io;   // half: pairs; lanes: of a head (with a norm a power of two: their sums cross lanes)
    float eps, amplitude;
};

constexpr int kTurnThreads = 256;

constexpr int kNormAny = 2;   // NORM: 0 none, 1 of heads whose squares lie in fp32's range or count for nothing beside eps, kNormAny of all
template <typename T, bool BACK, int NORM, bool PAIRS>
__global__ __launch_bounds__(kTurnThreads) void rotate_kernel(const TurnArgs a) {
    constexpr int kN = Frag<T>::kN;
    __shared__ float2 tables[4][64 * kN + kN];   // cosine and sine of the pairs of a wavefront's rows, times the amplitude
    __shared__ float join[BACK && NORM ? 4 : 1][256];
    const bool second = blockIdx.x >= a.part[0].blocks;
    const TurnPart& p = a.part[second];
    const uint32_t block = second ? blockIdx.x - a.part[0].blocks : blockIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id(), lanes = a.lanes, group = lane / lanes, l = lane - group * lanes;
    const int beside = p.beside, mine = group / beside;   // mine: this lane's of the wavefront's rows (`per` and more: none)
    // This lane's elements of a head: two runs of up to kN.  Pairs (j, j + half): the runs lie `half` apart, behind them the elements that are not
    // turned; pairs (2 j, 2 j + 1): the runs follow each other.
    int ea, eb, na, nb, first, again_a, again_b;   // first: number of the first pair
    if (PAIRS) {
        ea = 2 * kN * l;
        eb = ea + kN;
        na = a.dim - ea;
        nb = a.dim - eb;
        na = na < 0 ? 0 : (na < kN ? na : kN);
        nb = nb < 0 ? 0 : (nb < kN ? nb : kN);
        move_back(ea, na, again_a, 0, kN, true);
        move_back(eb, nb, again_b, 0, kN, true);
        first = ea / 2;   // (of the first run; of the second: below)
    } else {
        const int turning = (a.half + kN - 1) / kN;
        const bool turns = l < turning;
        ea = turns ? l * kN : 2 * a.half + 2 * kN * (l - turning);
        na = (turns ? a.half : a.dim) - ea;
        na = na < 0 ? 0 : (na < kN ? na : kN);
        eb = ea + kN;
        nb = a.dim - eb;
        nb = nb < 0 ? 0 : (nb < kN ? nb : kN);
        move_back(ea, na, again_a, turns ? 0 : 2 * a.half, kN, false);
        if (turns) {
            eb = a.half + ea;
            nb = na;
            again_b = again_a;
        } else {
            move_back(eb, nb, again_b, 2 * a.half, kN, false);
        }
        first = turns ? ea : a.half;   // (no pair)
    }
    const int first_b = PAIRS ? eb / 2 : first;
    float wa[kN], wb[kN], dwa[kN], dwb[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) {
        wa[j] = NORM && p.weight && j < na ? param_load(p.weight, a.param_io, ea + j) : 1.f;
        wb[j] = NORM && p.weight && j < nb ? param_load(p.weight, a.param_io, eb + j) : 1.f;
        dwa[j] = dwb[j] = 0.f;
    }
    const float inv = 1.f / (float)a.dim;
    const int pairs = a.half * p.per;   // of a wavefront's rows
    float2* const table = tables[wave];
    for (uint32_t u = block * 4 + wave; u < p.units; u += p.blocks * 4) {
        const uint32_t step = u / (uint32_t)p.pieces;
        const int piece = (int)(u - step * (uint32_t)p.pieces);
        const int64_t row0 = (int64_t)step * p.per, row = row0 + mine;
        const bool is = mine < p.per && row < a.rows;
        const int64_t at = is ? row : 0;
        int head = piece * p.turns * beside + group - mine * beside;
        uint4 first_in[NORM && BACK ? 4 : 2];   // the first turn's elements, under way beside the angles
        const auto load = [&](uint4 (&raw)[NORM && BACK ? 4 : 2]) __attribute__((always_inline)) {
            const bool here = is && head < p.heads;
            const int h0 = here ? head : 0, n0 = here ? na : 0, n1 = here ? nb : 0;
            const T* const from = static_cast<const T*>(BACK ? p.dy : p.x) + (BACK ? at * p.dy_row + h0 * p.dy_head : at * p.x_row + h0 * p.x_head);
            raw[0] = load_some<T>(from + ea, n0);
            raw[1] = load_some<T>(from + eb, n1);
            if constexpr (BACK && NORM) {
                const T* const in = static_cast<const T*>(p.x) + at * p.x_row + h0 * p.x_head;
                raw[2] = load_some<T>(in + ea, n0);
                raw[3] = load_some<T>(in + eb, n1);
            }
        };
        load(first_in);
        // The rows' pairs shared among the wavefront's lanes: of a row, as many lanes as there are heads beside each other would otherwise do the same.
        for (int n = lane; n < pairs; n += 64) {
            const int of = n / a.half, pair = n - of * a.half;
            const int64_t r = row0 + of < a.rows ? row0 + of : 0;
            const float2 cs = cos_sin((double)a.positions[r] * (a.frequencies[pair] * 0.15915494309189533577));   // (in turns)
            table[n] = make_float2(cs.x * a.amplitude, BACK ? -cs.y * a.amplitude : cs.y * a.amplitude);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        float2 cs[kN];   // (PAIRS: kN / 2 of either run)
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const int pair = PAIRS ? (j < kN / 2 ? first + j : first_b + j - kN / 2) : first + j;
            cs[j] = table[is ? mine * a.half + (pair < a.half ? pair : 0) : 0];
        }
        // (all lanes of a wavefront stay in the loop together: the sums across lanes need them)
        for (int k = 0; k < p.turns; ++k) {
            uint4 raw[NORM && BACK ? 4 : 2];
            if (k > 0) {
                load(raw);
            } else {
#pragma unroll
                for (int i = 0; i < (NORM && BACK ? 4 : 2); ++i) raw[i] = first_in[i];
            }
            const bool here = is && head < p.heads;
            float ua[kN], ub[kN], xa[kN], xb[kN];
            Frag<T>::unpack(raw[0], ua);
            Frag<T>::unpack(raw[1], ub);
            if constexpr (BACK && NORM) {
                Frag<T>::unpack(raw[2], xa);
                Frag<T>::unpack(raw[3], xb);
            }
            if constexpr (!BACK && NORM) {
                float by;
                const float r = head_rstd<NORM == kNormAny>(ua, ub, again_a, again_b, lanes, inv, a.eps, here, by);
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    ua[j] = ua[j] * by * r * wa[j];
                    ub[j] = ub[j] * by * r * wb[j];
                }
            }
            // (elements that are not turned are left as they are: 0 times a neighbour that is not finite is not 0)
            if constexpr (PAIRS) {
#pragma unroll
                for (int j = 0; j < kN; j += 2) {
                    turn(first + j / 2 < a.half, cs[j / 2], ua[j], ua[j + 1]);
                    turn(first_b + j / 2 < a.half, cs[(kN + j) / 2], ub[j], ub[j + 1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < kN; ++j) turn(first < a.half, cs[j], ua[j], ub[j]);
            }
            if constexpr (BACK && NORM) {
                float by, m = 0.f;
                float r = head_rstd<NORM == kNormAny>(xa, xb, again_a, again_b, lanes, inv, a.eps, here, by);
#pragma unroll
                for (int j = 0; j < kN; ++j) m = j < again_a ? m : fmaf(ua[j] * wa[j], xa[j] * by, m);
#pragma unroll
                for (int j = 0; j < kN; ++j) m = j < again_b ? m : fmaf(ub[j] * wb[j], xb[j] * by, m);
                r = here ? r : 0.f;
                m = group_sum(m, lanes) * inv * r;   // the mean of u h
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    const float ha = xa[j] * by * r, hb = xb[j] * by * r;
                    dwa[j] = fmaf(ua[j], ha, dwa[j]);
                    dwb[j] = fmaf(ub[j], hb, dwb[j]);
                    ua[j] = r * (ua[j] * wa[j] - ha * m) * by;
                    ub[j] = r * (ub[j] * wb[j] - hb * m) * by;
                }
            }
            T* const to = static_cast<T*>(p.y) + at * p.y_row + (here ? head : 0) * p.y_head;
            store_some<T>(to + ea, here ? na : 0, ua);
            store_some<T>(to + eb, here ? nb : 0, ub);
            head += beside;
        }
        __builtin_amdgcn_wave_barrier();   // (the next rows' pairs go where these are)
    }
    if constexpr (BACK && NORM) {
        if (!p.partial) return;
        // the groups of a wavefront, then the wavefronts, in a fixed order
        for (int w = lanes; w < 64; w <<= 1)
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                dwa[j] += __shfl_xor(dwa[j], w);
                dwb[j] += __shfl_xor(dwb[j], w);
            }
        if (group == 0) {
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                if (j >= again_a && j < na) join[wave][ea + j] = dwa[j];
                if (j >= again_b && j < nb) join[wave][eb + j] = dwb[j];
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < a.dim; e += kTurnThreads)
            p.partial[(int64_t)block * a.dim + e] = (join[0][e] + join[1][e]) + (join[2][e] + join[3][e]);
    }
}

// The weights' gradients from the workgroups' sums: 8 columns a workgroup, 32 slices of the workgroups beside each other; q's columns, then k's.
__global__ __launch_bounds__(256) void rotate_params_kernel(const float* __restrict__ partial, const int blocks_q, const int blocks_k, const int n, void* dq,
                                                            void* dk, const int io) {
    __shared__ float part[32][9];
    const int c = threadIdx.x % 8, k = threadIdx.x / 8, e = blockIdx.x * 8 + c;
    const bool second = e >= n;
    const float* const from = partial + (second ? (int64_t)blocks_q * n + (e - n) : e);
    part[k][c] = e < 2 * n ? strided_sum(from, n, k, second ? blocks_k : blocks_q, 32) : 0.f;
    __syncthreads();
    if (k == 0 && e < 2 * n) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += part[i][c];
        void* const to = second ? dk : dq;
        if (to) param_store(to, io, second ? e - n : e, t);
    }
}

static int turn_lanes(const int dim, const int half, const bool pairs, const int kN, const bool norm) {
    const int lanes = pairs ? (dim + 2 * kN - 1) / (2 * kN) : (half + kN - 1) / kN + (dim - 2 * half + 2 * kN - 1) / (2 * kN);
    int n = 1;
    while (n < lanes) n <<= 1;
    return norm ? n : lanes;
}
// How the heads of q or k are shared among wavefronts: some beside each other, the others one after the other with the same sines and cosines, unless
// there would be few wavefronts then.
static void turn_units(TurnPart& p, const int64_t rows, const int heads, const int lanes) {
    p.heads = heads;
    p.units = 0;
    p.pieces = p.turns = p.per = p.beside = 1;
    if (heads == 0) return;
    const HeadShare share = share_heads(64 / lanes, heads);
    p.beside = share.beside;
    p.per = share.per;
    const int64_t steps = (rows + p.per - 1) / p.per, all = (heads + p.beside - 1) / p.beside;
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(all, 8192 / std::max<int64_t>(1, steps)));
    p.turns = (int)((all + want - 1) / want);
    p.pieces = (int)((all + p.turns - 1) / p.turns);
    p.units = (uint32_t)(steps * p.pieces);
}
// Workgroups of q and of k: at most `most` in all, in proportion to their heads, so that they end together.
static void turn_blocks(TurnPart& q, TurnPart& k, const int64_t most) {
    const int64_t heads = q.heads + k.heads;
    const auto some = [&](const TurnPart& p) {
        return p.units == 0 ? 0u : (uint32_t)std::min<int64_t>(((int64_t)p.units + 3) / 4, std::max<int64_t>(1, most * p.heads / heads));
    };
    q.blocks = some(q);
    k.blocks = some(k);
}
// More of them than the chip holds at once: forward 1280 / 2048 / 8192 / 16384 workgroups 361 / 288 / 268 / 270 us (131,071 rows of 20 heads of 128
// bfloat16); backward 512 / 768 / 1024 / 2048 / 3584 / 4096 284 / 237 / 268 / 224 / 214 / 223 (65,537 rows), where each leaves sums to be added.
constexpr int64_t kTurnBlocksForward = 8192, kTurnBlocksBackward = 3584;

size_t rotate_workspace(const int dim) {   // (of any element type and layout)
    return (((size_t)kTurnBlocksBackward + 2) * (size_t)dim * sizeof(float) + 255) & ~(size_t)255;
}

template <typename T, bool BACK, int NORM>
static void launch_layout(const TurnArgs& a, const bool pairs, const unsigned blocks, hipStream_t s) {
    if (pairs) rotate_kernel<T, BACK, NORM, true><<<blocks, kTurnThreads, 0, s>>>(a);
    else rotate_kernel<T, BACK, NORM, false><<<blocks, kTurnThreads, 0, s>>>(a);
}
template <typename T, bool BACK>
static void launch_norm(const TurnArgs& a, const bool norm, const bool pairs, const unsigned blocks, hipStream_t s) {
    if (norm && a.eps < kEpsAny) launch_layout<T, BACK, kNormAny>(a, pairs, blocks, s);
    else if (norm) launch_layout<T, BACK, 1>(a, pairs, blocks, s);
    else launch_layout<T, BACK, 0>(a, pairs, blocks, s);
}
template <typename T>
static void launch_turn(const TurnArgs& a, const bool back, const bool norm, const bool pairs, const unsigned blocks, hipStream_t s) {
    if (back) launch_norm<T, true>(a, norm, pairs, blocks, s);
    else launch_norm<T, false>(a, norm, pairs, blocks, s);
}

hipError_t launch_rotate(const tbe_handle* h, const RotateCall& r, const bool back, hipStream_t s) {
    TurnArgs a{};
    a.positions = IdxView{r.positions, r.positions32};
    a.frequencies = r.frequencies;
    a.rows = r.rows; a.dim = r.dim; a.half = r.turned / 2; a.param_io = r.param_io;
    a.eps = r.eps; a.amplitude = r.amplitude;
    a.lanes = turn_lanes(r.dim, a.half, r.pairs, r.io == 0 ? 4 : 8, r.norm);
    for (int i = 0; i < 2; ++i) {
        const RotateMatrix& m = r.part[i];
        TurnPart& p = a.part[i];
        p.x = m.x.data; p.x_row = m.x.row_stride; p.x_head = m.x.head_stride;
        p.dy = m.dy.data; p.dy_row = m.dy.row_stride; p.dy_head = m.dy.head_stride;
        p.y = m.y.data; p.y_row = m.y.row_stride; p.y_head = m.y.head_stride;
        p.weight = m.weight;
        turn_units(p, r.rows, m.heads, a.lanes);
    }
    turn_blocks(a.part[0], a.part[1], back ? kTurnBlocksBackward : kTurnBlocksForward);
    const bool weights = back && r.norm && (r.part[0].dw || r.part[1].dw);
    if (weights) {
        a.part[0].partial = static_cast<float*>(r.workspace);
        a.part[1].partial = a.part[0].partial + (size_t)a.part[0].blocks * r.dim;
    }
    const unsigned blocks = a.part[0].blocks + a.part[1].blocks;
    if (blocks > 0) {
        LaunchTimer tm(h, s, back ? "rotate_backward" : "rotate");
        if (r.io == 0) launch_turn<float>(a, back, r.norm, r.pairs, blocks, s);
        else if (r.io == 1) launch_turn<__half>(a, back, r.norm, r.pairs, blocks, s);
        else launch_turn<bf16_t>(a, back, r.norm, r.pairs, blocks, s);
        tm.done();
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!weights) return hipSuccess;
    LaunchTimer tp(h, s, "rotate_params");
    rotate_params_kernel<<<(2 * r.dim + 7) / 8, 256, 0, s>>>(a.part[0].partial, (int)a.part[0].blocks, (int)a.part[1].blocks, r.dim, r.part[0].dw, r.part[1].dw,
                                                             r.param_io);
    tp.done();
    return hipGetLastError();
}

}  // namespace tbe
