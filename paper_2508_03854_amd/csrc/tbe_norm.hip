// Layer norm over the last axis and its gradients.
//   forward   mean = 1/n sum x,  rstd = 1 / sqrt(1/n sum (x - mean)^2 + eps),  y = (x - mean) rstd w + b
//   backward  h = (x - mean) rstd,  g = dy w:   dx = rstd (g - 1/n sum g - h 1/n sum g h),  dw = sum over rows of dy h,  db = sum of dy
// Bound: the stream, every element read once and written once; a row stays in registers between its sums and its use.  The sums are
// in fp32, the variance from the differences to the mean (no difference of large squares); each result is rounded once.  Measured: 1,000,003
// rows of 128 bfloat16 forward 105 us, 5.0 TB/s; 262,147 of 256 backward 89 and 5 us for the sums over rows, 4.5 TB/s; 8001 of 1021 fp32
// backward 23 and 7 us.
#include <hip/hip_runtime.h>

#include "tbe_elems.h"
#include "tbe_internal.h"

namespace tbe {

// A row is shared by G lanes (a power of two up to a wavefront, or a whole workgroup), F fragments of sixteen bytes each: at most 32
// elements a lane.  Fragment f of lane l begins at element (f * G + l) * kN.
template <typename T, int F>
struct RowRegs {
    static constexpr int kN = Frag<T>::kN;
    uint4 raw[F];
    __device__ __forceinline__ void load(const T* row, const int n, const int l, const int G) {
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int e = (f * G + l) * kN;
            raw[f] = make_uint4(0u, 0u, 0u, 0u);
            if (e + kN <= n) {
                raw[f] = Frag<T>::load(row + e);
            } else if (e < n) {   // the row's last elements, one by one: nothing behind the row is read
                uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int i = 0; i < kN - 1; ++i)
                    if (e + i < n) {
                        if constexpr (kN == 4) w[i] = __float_as_uint(row[e + i]);
                        else w[i / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(row)[e + i] << (16 * (i % 2));
                    }
                raw[f] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
};
template <typename T, int F>
__device__ __forceinline__ void row_store(T* row, const int n, const int l, const int G, const float (&y)[F][Frag<T>::kN]) {
    constexpr int kN = Frag<T>::kN;
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int e = (f * G + l) * kN;
        if (e + kN <= n) {
            Frag<T>::store(row + e, y[f]);
        } else if (e < n) {
#pragma unroll
            for (int i = 0; i < kN - 1; ++i)
                if (e + i < n) row[e + i] = elem_round<T>(y[f][i]);
        }
    }
}
template <int F, int kN>
__device__ __forceinline__ void load_params(const void* p, const int io, const float none, const int n, const int l, const int G, float (&w)[F][kN]) {
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int e = (f * G + l) * kN + i;
            w[f][i] = p && e < n ? param_load(p, io, e) : none;
        }
}

constexpr int kNormThreads = 256;

// Sums over the lanes of a row, of two values at once; `both`: 2 * 4 floats of LDS, used where a row is the workgroup's (then a
// barrier on either side, so all of the workgroup comes here together).
template <int G>
__device__ __forceinline__ float2 row_sums(float a, float b, float* both) {
    if constexpr (G <= 64) {
        return make_float2(group_sum(a, G), group_sum(b, G));
    } else {
        a = group_sum(a, 64);
        b = group_sum(b, 64);
        __syncthreads();
        if (lane_id() == 0) {
            both[threadIdx.x >> 6] = a;
            both[4 + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        return make_float2(both[0] + both[1] + both[2] + both[3], both[4] + both[5] + both[6] + both[7]);
    }
}

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void* y;   // dx in the backward
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    float* partial;   // [workgroups][2][n]
    int64_t rows, x_stride, dy_stride, y_stride;
    int n, param_io;
    float eps;
};

template <typename T, int G, int F>
__global__ __launch_bounds__(kNormThreads) void layer_norm_kernel(const NormArgs a) {
    constexpr int kN = Frag<T>::kN, kPer = kNormThreads / G;   // rows of a workgroup at a time
    __shared__ float both[8];
    const int l = threadIdx.x % G, n = a.n;
    const float inv = 1.0f / (float)n;
    float w[F][kN], b[F][kN];
    load_params<F, kN>(a.weight, a.param_io, 1.f, n, l, G, w);
    load_params<F, kN>(a.bias, a.param_io, 0.f, n, l, G, b);
    // (all lanes of a wavefront stay in the loop together: the sums across lanes need them)
    for (int64_t r0 = (int64_t)blockIdx.x * kPer; r0 < a.rows; r0 += (int64_t)gridDim.x * kPer) {
        const int64_t r = r0 + threadIdx.x / G;
        const bool is = r < a.rows;
        RowRegs<T, F> in;
        in.load(static_cast<const T*>(a.x) + (is ? r : 0) * a.x_stride, is ? n : 0, l, G);
        float x[F][kN], s = 0.f;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            Frag<T>::unpack(in.raw[f], x[f]);
#pragma unroll
            for (int i = 0; i < kN; ++i) s += x[f][i];
        }
        const float mean = row_sums<G>(s, 0.f, both).x / (float)n;   // (a division: a constant row's mean is its value wherever n times it is exact)
        float q = 0.f;
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                x[f][i] = (f * G + l) * kN + i < n ? x[f][i] - mean : 0.f;
                q = fmaf(x[f][i], x[f][i], q);
            }
        const float rstd = 1.0f / sqrtf(row_sums<G>(q, 0.f, both).x * inv + a.eps);
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int i = 0; i < kN; ++i) x[f][i] = fmaf(x[f][i] * rstd, w[f][i], b[f][i]);
        if (is) {
            row_store<T, F>(static_cast<T*>(a.y) + r * a.y_stride, n, l, G, x);
            if (l == 0) {
                if (a.mean) a.mean[r] = mean;
                if (a.rstd) a.rstd[r] = rstd;
            }
        }
    }
}

// Every lane adds up dw and db of its columns over the rows it meets; the row groups of a workgroup are joined in LDS in a fixed
// order, the workgroups by norm_params_kernel: the sums do not depend on timing.
template <typename T, int G, int F>
__global__ __launch_bounds__(kNormThreads) void layer_norm_backward_kernel(const NormArgs a) {
    constexpr int kN = Frag<T>::kN, kPer = kNormThreads / G;
    __shared__ float both[8];
    extern __shared__ float join[];   // [2][n]
    const int l = threadIdx.x % G, n = a.n;
    const float inv = 1.0f / (float)n;
    float w[F][kN], dw[F][kN], db[F][kN];
    load_params<F, kN>(a.weight, a.param_io, 1.f, n, l, G, w);
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
        for (int i = 0; i < kN; ++i) dw[f][i] = db[f][i] = 0.f;
    for (int64_t r0 = (int64_t)blockIdx.x * kPer; r0 < a.rows; r0 += (int64_t)gridDim.x * kPer) {
        const int64_t r = r0 + threadIdx.x / G;
        const bool is = r < a.rows;
        const int64_t at = is ? r : 0;
        RowRegs<T, F> in, up;
        in.load(static_cast<const T*>(a.x) + at * a.x_stride, is ? n : 0, l, G);
        up.load(static_cast<const T*>(a.dy) + at * a.dy_stride, is ? n : 0, l, G);
        const float mean = a.mean_in[at], rstd = is ? a.rstd_in[at] : 0.f;
        float h[F][kN], g[F][kN], sg = 0.f, sh = 0.f;
#pragma unroll
        for (int f = 0; f < F; ++f) {
            Frag<T>::unpack(in.raw[f], h[f]);
            Frag<T>::unpack(up.raw[f], g[f]);
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                h[f][i] = is && (f * G + l) * kN + i < n ? (h[f][i] - mean) * rstd : 0.f;
                dw[f][i] = fmaf(g[f][i], h[f][i], dw[f][i]);
                db[f][i] += g[f][i];
                g[f][i] *= w[f][i];
                sg += g[f][i];
                sh = fmaf(g[f][i], h[f][i], sh);
            }
        }
        const float2 s = row_sums<G>(sg, sh, both);
        const float mg = s.x * inv, mh = s.y * inv;
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int i = 0; i < kN; ++i) g[f][i] = (g[f][i] - mg - h[f][i] * mh) * rstd;
        if (is) row_store<T, F>(static_cast<T*>(a.y) + r * a.y_stride, n, l, G, g);
    }
    if (!a.partial) return;
    if constexpr (kPer > 1) {
        for (int k = 0; k < kPer; ++k) {   // row group k adds its sums
            if ((int)threadIdx.x / G == k) {
#pragma unroll
                for (int f = 0; f < F; ++f)
#pragma unroll
                    for (int i = 0; i < kN; ++i) {
                        const int e = (f * G + l) * kN + i;
                        if (e < n) {
                            join[e] = k ? join[e] + dw[f][i] : dw[f][i];
                            join[n + e] = k ? join[n + e] + db[f][i] : db[f][i];
                        }
                    }
            }
            __syncthreads();
        }
        for (int e = threadIdx.x; e < 2 * n; e += kNormThreads) a.partial[(int64_t)blockIdx.x * 2 * n + e] = join[e];
    } else {
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const int e = (f * G + l) * kN + i;
                if (e < n) {
                    a.partial[(int64_t)blockIdx.x * 2 * n + e] = dw[f][i];
                    a.partial[(int64_t)blockIdx.x * 2 * n + n + e] = db[f][i];
                }
            }
    }
}

// Columns of the weight's and the bias's gradient: 8 columns a workgroup, 32 slices of the workgroups' sums beside each other.
__global__ __launch_bounds__(256) void norm_params_kernel(const float* __restrict__ partial, const int blocks, const int n, void* dw, void* db, const int io) {
    __shared__ float part[32][9];
    const int c = threadIdx.x % 8, k = threadIdx.x / 8, e = blockIdx.x * 8 + c;
    part[k][c] = e < 2 * n ? strided_sum(partial + e, 2 * n, k, blocks, 32) : 0.f;
    __syncthreads();
    if (k == 0 && e < 2 * n) {
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += part[i][c];
        void* const to = e < n ? dw : db;
        if (to) param_store(to, io, e < n ? e : e - n, t);
    }
}

// How a row of n elements is shared: the fewest lanes that hold it in one fragment each, then a wavefront with up to 32 elements a lane, then a
// workgroup: from three quarters of its lanes on, since fewer registers a lane leave room for more rows under way.  Wavefront / workgroup, us,
// forward and backward: 20,000 x 1024 fp32 34 / 31, 61 / 50; 30,000 x 800 38 / 39.5, 80 / 70; with fewer lanes busy 60,000 x 700 61 / 80, 124 /
// 139, 60,000 x 1000 bfloat16 59 / 91, 95 / 146.
struct NormShape {
    int lanes, frags;
};
static NormShape norm_shape(const int n, const int kN) {
    const int frags = (n + kN - 1) / kN;
    if (frags <= 64) {
        int G = 4;
        while (G < frags) G <<= 1;
        return {G, 1};
    }
    for (int F = 2; F * kN <= 32; F <<= 1)
        if (frags <= 64 * F && n <= 1024 && frags <= 192) return {64, F};
    for (int F = 1;; F <<= 1)
        if (frags <= 256 * F) return {256, F};
}

// Workgroups: no more than the chip holds at once, so that none comes late, by the registers that a lane's elements take.  Backward, 1024 / this,
// us: 60,000 x 700 fp32 168 / 126, 60,000 x 1000 bfloat16 132 / 97.
static int norm_blocks(const int64_t rows, const int n, const int kN, const bool backward) {
    const NormShape sh = norm_shape(n, kN);
    const int64_t turns = (rows * sh.lanes + kNormThreads - 1) / kNormThreads;   // of one workgroup
    const int each = sh.frags * kN;
    const int64_t most = 256 * (backward ? (each <= 8 ? 4 : (each <= 16 ? 3 : 1)) : (each <= 8 ? 8 : (each <= 16 ? 5 : 2)));
    return (int)(turns < 1 ? 1 : turns < most ? turns : most);
}
size_t layer_norm_workspace(const int64_t rows, const int n) {   // (of any element type)
    const int a = norm_blocks(rows, n, 4, true), b = norm_blocks(rows, n, 8, true);
    return ((size_t)(a > b ? a : b) * 2 * (size_t)n * sizeof(float) + 255) & ~(size_t)255;
}

template <typename T, int G, int F>
static void launch_shape(const NormArgs& a, const bool backward, const int blocks, hipStream_t s) {
    if (backward) layer_norm_backward_kernel<T, G, F><<<blocks, kNormThreads, G < kNormThreads ? 2 * (size_t)a.n * sizeof(float) : 0, s>>>(a);
    else layer_norm_kernel<T, G, F><<<blocks, kNormThreads, 0, s>>>(a);
}
template <typename T>
static void launch_norm(const NormArgs& a, const bool backward, hipStream_t s) {
    constexpr int kN = Frag<T>::kN;
    const NormShape sh = norm_shape(a.n, kN);
    const int blocks = norm_blocks(a.rows, a.n, kN, backward);
    switch (sh.lanes * 16 + sh.frags) {
        case 4 * 16 + 1: return launch_shape<T, 4, 1>(a, backward, blocks, s);
        case 8 * 16 + 1: return launch_shape<T, 8, 1>(a, backward, blocks, s);
        case 16 * 16 + 1: return launch_shape<T, 16, 1>(a, backward, blocks, s);
        case 32 * 16 + 1: return launch_shape<T, 32, 1>(a, backward, blocks, s);
        case 64 * 16 + 1: return launch_shape<T, 64, 1>(a, backward, blocks, s);
        case 64 * 16 + 2: return launch_shape<T, 64, 2>(a, backward, blocks, s);
        case 64 * 16 + 4: if constexpr (kN == 4) return launch_shape<T, 64, 4>(a, backward, blocks, s); else return;
        case 256 * 16 + 1: return launch_shape<T, 256, 1>(a, backward, blocks, s);
        case 256 * 16 + 2: return launch_shape<T, 256, 2>(a, backward, blocks, s);
        case 256 * 16 + 4: return launch_shape<T, 256, 4>(a, backward, blocks, s);
        case 256 * 16 + 8: if constexpr (kN == 4) return launch_shape<T, 256, 8>(a, backward, blocks, s); else return;
    }
}
static void launch_norm_io(const NormArgs& a, const int io, const bool backward, hipStream_t s) {
    if (io == 0) launch_norm<float>(a, backward, s);
    else if (io == 1) launch_norm<__half>(a, backward, s);
    else launch_norm<bf16_t>(a, backward, s);
}

hipError_t launch_layer_norm(const tbe_handle* h, const void* x, int64_t x_stride, int io, int64_t rows, int n, const void* weight,
                             const void* bias, int param_io, float eps, void* y, int64_t y_stride, float* mean, float* rstd, hipStream_t s) {
    NormArgs a{};
    a.x = x; a.x_stride = x_stride; a.rows = rows; a.n = n;
    a.weight = weight; a.bias = bias; a.param_io = param_io; a.eps = eps;
    a.y = y; a.y_stride = y_stride; a.mean = mean; a.rstd = rstd;
    LaunchTimer tm(h, s, "layer_norm");
    launch_norm_io(a, io, false, s);
    tm.done();
    return hipGetLastError();
}

hipError_t launch_layer_norm_backward(const tbe_handle* h, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int io,
                                      int64_t rows, int n, const void* weight, int param_io, const float* mean, const float* rstd,
                                      void* dx, int64_t dx_stride, void* dw, void* db, void* workspace, hipStream_t s) {
    NormArgs a{};
    a.x = x; a.x_stride = x_stride; a.dy = dy; a.dy_stride = dy_stride; a.rows = rows; a.n = n;
    a.weight = weight; a.param_io = param_io; a.mean_in = mean; a.rstd_in = rstd;
    a.y = dx; a.y_stride = dx_stride;
    a.partial = dw || db ? static_cast<float*>(workspace) : nullptr;
    LaunchTimer tm(h, s, "layer_norm_backward");
    launch_norm_io(a, io, true, s);
    tm.done();
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.partial) return e;
    LaunchTimer tp(h, s, "layer_norm_params");
    norm_params_kernel<<<(2 * n + 7) / 8, 256, 0, s>>>(a.partial, norm_blocks(rows, n, io == 0 ? 4 : 8, true), n, dw, db, param_io);
    tp.done();
    return hipGetLastError();
}

}  // namespace tbe
