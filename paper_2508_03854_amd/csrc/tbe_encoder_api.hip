// C ABI of the operators on sequences of looked-up rows: argument checks, workspaces.  Nothing is launched when a check fails.
#include <math.h>

#include "tbe_attention.h"

using namespace tbe;

static bool multiple_of(const void* p, const size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
static bool io_known(const int io) { return io == TBE_IO_F32 || io == TBE_IO_F16 || io == TBE_IO_BF16; }
static size_t io_size(const tbe_io_dtype io) { return io == TBE_IO_F32 ? 4 : 2; }
static tbe_status done(const hipError_t e) { return e == hipSuccess ? TBE_OK : TBE_EHIP; }

extern "C" {

static tbe_status check_norm(const tbe_handle* h, const int64_t rows, const int32_t cols) {
    if (!h) return TBE_EINVAL;
    return rows < 0 || rows >= ((int64_t)1 << 31) || cols < 1 || cols > kNormMaxCols ? TBE_ESHAPE : TBE_OK;
}
// a matrix of `rows` rows, `stride` elements apart
static bool matrix_ok(const void* p, const int64_t stride, const int64_t rows, const int32_t cols, const size_t size) {
    return (p || rows == 0) && multiple_of(p, size) && (stride >= cols || rows <= 1) && stride < ((int64_t)1 << 40);
}

tbe_status tbe_layer_norm(const tbe_handle* h, const void* x, int64_t x_stride, tbe_io_dtype dtype, int64_t rows, int32_t cols,
                          const void* weight, const void* bias, tbe_io_dtype param_dtype, float eps, void* y, int64_t y_stride,
                          float* mean, float* rstd, void* hip_stream) {
    const tbe_status st = check_norm(h, rows, cols);
    if (st != TBE_OK) return st;
    if (!io_known(dtype) || !io_known(param_dtype)) return TBE_EDTYPE;
    const size_t e = io_size(dtype), p = io_size(param_dtype);
    if (!matrix_ok(x, x_stride, rows, cols, e) || !matrix_ok(y, y_stride, rows, cols, e)) return TBE_EINVAL;
    if (!multiple_of(weight, p) || !multiple_of(bias, p) || !multiple_of(mean, 4) || !multiple_of(rstd, 4)) return TBE_EINVAL;
    if (!isfinite(eps) || eps < 0.f || (x == y && x_stride != y_stride && rows > 1)) return TBE_EINVAL;
    if (rows == 0) return TBE_OK;
    return done(launch_layer_norm(h, x, x_stride, (int)dtype, rows, cols, weight, bias, (int)param_dtype, eps, y, y_stride, mean, rstd,
                                  static_cast<hipStream_t>(hip_stream)));
}

tbe_status tbe_layer_norm_workspace_bytes(const tbe_handle* h, int64_t rows, int32_t cols, size_t* bytes) {
    if (!bytes) return TBE_EINVAL;
    const tbe_status st = check_norm(h, rows, cols);
    if (st == TBE_OK) *bytes = layer_norm_workspace(rows, cols);
    return st;
}

tbe_status tbe_layer_norm_backward(const tbe_handle* h, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride,
                                   tbe_io_dtype dtype, int64_t rows, int32_t cols, const void* weight, tbe_io_dtype param_dtype,
                                   const float* mean, const float* rstd, void* dx, int64_t dx_stride, void* dweight, void* dbias,
                                   void* workspace, size_t workspace_bytes, void* hip_stream) {
    const tbe_status st = check_norm(h, rows, cols);
    if (st != TBE_OK) return st;
    if (!io_known(dtype) || !io_known(param_dtype)) return TBE_EDTYPE;
    const size_t e = io_size(dtype), p = io_size(param_dtype);
    if (!matrix_ok(dy, dy_stride, rows, cols, e) || !matrix_ok(x, x_stride, rows, cols, e) || !matrix_ok(dx, dx_stride, rows, cols, e)) return TBE_EINVAL;
    if (((!mean || !rstd) && rows > 0) || !multiple_of(mean, 4) || !multiple_of(rstd, 4)) return TBE_EINVAL;
    if (!multiple_of(weight, p) || !multiple_of(dweight, p) || !multiple_of(dbias, p)) return TBE_EINVAL;
    if (rows > 1 && ((dx == dy && dx_stride != dy_stride) || (dx == x && dx_stride != x_stride))) return TBE_EINVAL;
    if (dweight || dbias) {
        if (!workspace || !multiple_of(workspace, 256)) return TBE_EINVAL;
        if (workspace_bytes < layer_norm_workspace(rows, cols)) return TBE_EWORKSPACE;
    } else if (rows == 0) {
        return TBE_OK;
    }
    return done(launch_layer_norm_backward(h, dy, dy_stride, x, x_stride, (int)dtype, rows, cols, weight, (int)param_dtype, mean, rstd, dx,
                                           dx_stride, dweight, dbias, workspace, static_cast<hipStream_t>(hip_stream)));
}

static tbe_status check_attention_sizes(const tbe_handle* h, const tbe_attention_args* a) {
    if (!h || !a) return TBE_EINVAL;
    if (!io_known(a->dtype) || (a->index_dtype != TBE_I64 && a->index_dtype != TBE_I32)) return TBE_EDTYPE;
    const int64_t most = ((int64_t)1 << 31) - 4096;   // (a tile beyond the last row has a number still)
    if (a->sequences < 1 || a->sequences >= 1 << 24 || a->q_rows < 0 || a->q_rows > most || a->k_rows < 0 || a->k_rows > most) return TBE_ESHAPE;
    if (a->kv_heads < 1 || a->heads < a->kv_heads || a->heads > 1024 || a->heads % a->kv_heads != 0) return TBE_ESHAPE;
    if (a->head_dim < 1 || a->head_dim > kAttnMaxDim || a->head_dim % (16 / (int)io_size(a->dtype)) != 0) return TBE_ESHAPE;
    if (a->buckets < 0 || a->buckets > 1024) return TBE_ESHAPE;
    return TBE_OK;
}
static AttnShape attention_shape(const tbe_attention_args* a) {
    AttnShape sh;
    sh.q_rows = a->q_rows; sh.k_rows = a->k_rows;
    sh.N = a->sequences; sh.H = a->heads; sh.kv = a->kv_heads; sh.dim = a->head_dim;
    sh.buckets = a->bias ? a->buckets : 0; sh.far = a->max_distance; sh.caches = a->k_lengths != nullptr;
    sh.narrow = a->dtype != TBE_IO_F32;
    return sh;
}
// the kernels' view of a matrix; false: not as it has to be
static bool rows_view(const tbe_rows& m, const int64_t rows, const int32_t heads, const tbe_attention_args* a, const bool result, RowsView& v) {
    const int64_t e = (int64_t)io_size(a->dtype);
    if (!m.data && rows > 0) return false;
    if (!multiple_of(m.data, 16) || m.row_stride < 0 || m.row_stride >= 1 << 22 || m.row_stride * e % 16 != 0) return false;
    if (m.head_stride < 0 || m.head_stride >= (int64_t)1 << 40 || m.head_stride * e % 16 != 0) return false;
    if (result && ((rows > 1 && m.row_stride < a->head_dim) || (rows > 0 && heads > 1 && m.head_stride < a->head_dim))) return false;   // (two writers of one element)
    v.p = static_cast<const char*>(m.data); v.row = m.row_stride * e; v.head = m.head_stride * e;
    return true;
}
static tbe_status attention_args(const tbe_handle* h, const tbe_attention_args* a, AttnArgs& k) {
    const tbe_status st = check_attention_sizes(h, a);
    if (st != TBE_OK) return st;
    if (a->bias && !io_known(a->bias_dtype)) return TBE_EDTYPE;
    if (a->bias && (a->buckets < 1 || a->max_distance < 0 || a->max_distance > kAttnMaxFar)) return TBE_ESHAPE;
    if (a->bias && (!multiple_of(a->bias, io_size(a->bias_dtype)) || !a->bucket_map || !multiple_of(a->bucket_map, 4))) return TBE_EINVAL;
    const size_t ia = a->index_dtype == TBE_I32 ? 4 : 8;
    if (!a->q_offsets || !a->k_offsets || !multiple_of(a->q_offsets, ia) || !multiple_of(a->k_offsets, ia) || !multiple_of(a->k_lengths, ia)) return TBE_EINVAL;
    if (!isfinite(a->scale)) return TBE_EINVAL;
    k = AttnArgs{};
    if (!rows_view(a->q, a->q_rows, a->heads, a, false, k.q) || !rows_view(a->k, a->k_rows, a->kv_heads, a, false, k.k) ||
        !rows_view(a->v, a->k_rows, a->kv_heads, a, false, k.v)) return TBE_EINVAL;
    const int is32 = a->index_dtype == TBE_I32;
    k.q_off = IdxView{a->q_offsets, is32}; k.k_off = IdxView{a->k_offsets, is32}; k.k_len = IdxView{a->k_lengths, is32};
    k.N = a->sequences; k.H = a->heads; k.kv = a->kv_heads; k.group = a->heads / a->kv_heads; k.dim = a->head_dim; k.causal = a->causal != 0;
    k.q_rows = a->q_rows; k.k_rows = a->k_rows;
    k.scale = a->scale; k.negative = a->scale < 0.f;
    // (a scale of 0 would make NaN of what is masked by -infinity; the smallest number makes all scores 0 as well)
    const float mag = fabsf(a->scale) * kLog2e;
    if (!isfinite(mag)) return TBE_EINVAL;
    k.scale2 = mag < 1.17549435e-38f ? 1.17549435e-38f : mag;
    if (a->bias) {
        k.bias = a->bias; k.bias_io = (int)a->bias_dtype; k.buckets = a->buckets; k.map = a->bucket_map; k.far = a->max_distance;
    }
    k.err = h->d_err;
    return TBE_OK;
}

tbe_status tbe_attention_workspace_bytes(const tbe_handle* h, const tbe_attention_args* args, int backward, size_t* bytes) {
    if (!bytes) return TBE_EINVAL;
    const tbe_status st = check_attention_sizes(h, args);
    if (st != TBE_OK) return st;
    AttnShape sh = attention_shape(args);
    sh.buckets = args->buckets;
    *bytes = attn_workspace(sh, backward != 0);
    return TBE_OK;
}

tbe_status tbe_attention(const tbe_handle* h, const tbe_attention_args* args, tbe_rows out, float* lse, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
    AttnArgs k;
    const tbe_status st = attention_args(h, args, k);
    if (st != TBE_OK) return st;
    if (!rows_view(out, args->q_rows, args->heads, args, true, k.o) || !multiple_of(lse, 4)) return TBE_EINVAL;
    k.lse = lse;
    const AttnShape sh = attention_shape(args);
    const AttnPlan p = attn_plan(sh);
    const size_t need = p.part_ml + p.part_o;
    if (need > 0) {
        if (!workspace || !multiple_of(workspace, 256)) return TBE_EINVAL;
        if (workspace_bytes < need) return TBE_EWORKSPACE;
    }
    if (!attn_grid_ok(sh, p)) return TBE_ESHAPE;
    if (args->q_rows == 0) return TBE_OK;
    return done(launch_attention(h, k, p, (int)args->dtype, workspace, static_cast<hipStream_t>(hip_stream)));
}

tbe_status tbe_attention_backward(const tbe_handle* h, const tbe_attention_args* args, tbe_rows out, const float* lse, tbe_rows dout,
                                  tbe_rows dq, tbe_rows dk, tbe_rows dv, void* dbias, void* workspace, size_t workspace_bytes,
                                  void* hip_stream) {
    AttnArgs k;
    const tbe_status st = attention_args(h, args, k);
    if (st != TBE_OK) return st;
    if (!rows_view(out, args->q_rows, args->heads, args, false, k.o) || !rows_view(dout, args->q_rows, args->heads, args, false, k.dout)) return TBE_EINVAL;
    if (!rows_view(dq, args->q_rows, args->heads, args, true, k.dq) || !rows_view(dk, args->k_rows, args->kv_heads, args, true, k.dk) ||
        !rows_view(dv, args->k_rows, args->kv_heads, args, true, k.dv)) return TBE_EINVAL;
    if ((!lse && args->q_rows > 0) || !multiple_of(lse, 4)) return TBE_EINVAL;
    if (dbias && (!args->bias || !multiple_of(dbias, io_size(args->bias_dtype)))) return TBE_EINVAL;
    k.lse = const_cast<float*>(lse);
    const AttnBackwardPlan p = attn_backward_plan(attention_shape(args));
    const size_t need = p.delta + p.part_bias + p.part_kv;
    if (need > 0) {
        if (!workspace || !multiple_of(workspace, 256)) return TBE_EINVAL;
        if (workspace_bytes < need) return TBE_EWORKSPACE;
    }
    if (!p.grid_ok) return TBE_ESHAPE;
    return done(launch_attention_backward(h, k, p, (int)args->dtype, dbias, workspace, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
