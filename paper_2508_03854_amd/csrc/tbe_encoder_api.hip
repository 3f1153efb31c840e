// C ABI of the operators on sequences of looked-up rows: argument checks, workspaces.  Nothing is launched when a check fails.
#include <math.h>

#include "tbe_attention.h"
#include "tbe_cache.h"
#include "tbe_overlap.h"

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
    if (result && rows > 0 && !runs_apart(HeadRuns{m.data, m.row_stride, m.head_stride, rows, heads, a->head_dim})) return false;
    v.p = static_cast<const char*>(m.data); v.row = m.row_stride * e; v.head = m.head_stride * e;
    return true;
}
static tbe_status attention_args(const tbe_handle* h, const tbe_attention_args* a, AttnArgs& k, const bool keys = true) {
    const tbe_status st = check_attention_sizes(h, a);
    if (st != TBE_OK) return st;
    if (a->bias && !io_known(a->bias_dtype)) return TBE_EDTYPE;
    if (a->bias && (a->buckets < 1 || a->max_distance < 0 || a->max_distance > kAttnMaxFar)) return TBE_ESHAPE;
    if (a->bias && (!multiple_of(a->bias, io_size(a->bias_dtype)) || !a->bucket_map || !multiple_of(a->bucket_map, 4))) return TBE_EINVAL;
    const size_t ia = a->index_dtype == TBE_I32 ? 4 : 8;
    if (!a->q_offsets || !a->k_offsets || !multiple_of(a->q_offsets, ia) || !multiple_of(a->k_offsets, ia) || !multiple_of(a->k_lengths, ia)) return TBE_EINVAL;
    if (!isfinite(a->scale)) return TBE_EINVAL;
    k = AttnArgs{};
    if (!rows_view(a->q, a->q_rows, a->heads, a, false, k.q)) return TBE_EINVAL;
    if (keys && (!rows_view(a->k, a->k_rows, a->kv_heads, a, false, k.k) || !rows_view(a->v, a->k_rows, a->kv_heads, a, false, k.v))) return TBE_EINVAL;
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

static tbe_status check_rotation(const tbe_handle* h, const tbe_rotation_args* a) {
    if (!h || !a) return TBE_EINVAL;
    if (!io_known(a->dtype) || (a->index_dtype != TBE_I64 && a->index_dtype != TBE_I32)) return TBE_EDTYPE;
    if (a->rows < 0 || a->rows >= (int64_t)1 << 31 || a->q_heads < 0 || a->q_heads > 1024 || a->k_heads < 0 || a->k_heads > 1024) return TBE_ESHAPE;
    if (a->q_heads + a->k_heads == 0 || a->head_dim < 1 || a->head_dim > kRotateMaxDim) return TBE_ESHAPE;
    return a->rotary_dim < 0 || a->rotary_dim > a->head_dim || a->rotary_dim % 2 != 0 ? TBE_ESHAPE : TBE_OK;
}
// a matrix of heads at any element's address
static bool loose_rows_ok(const tbe_rows& m, const tbe_rotation_args* a, const int32_t heads) {
    if (heads == 0 || a->rows == 0) return true;
    const auto stride_ok = [](const int64_t s) { return s >= 0 && s < (int64_t)1 << 40; };
    return m.data && multiple_of(m.data, io_size(a->dtype)) && stride_ok(m.row_stride) && stride_ok(m.head_stride);
}
// ... that is written: no element twice, and as its source where it is that
static bool loose_result_ok(const tbe_rows& m, const tbe_rotation_args* a, const int32_t heads) {
    if (!loose_rows_ok(m, a, heads)) return false;
    return heads == 0 || a->rows == 0 || runs_apart(HeadRuns{m.data, m.row_stride, m.head_stride, a->rows, heads, a->head_dim});
}
static HeadRuns runs_of(const tbe_rows& m, const tbe_rotation_args* a, const int32_t heads) {
    const int64_t e = (int64_t)io_size(a->dtype);
    return HeadRuns{m.data, m.row_stride * e, m.head_stride * e, a->rows, heads, a->head_dim * e};
}
static bool apart(const tbe_rows& x, const int32_t x_heads, const tbe_rows& y, const int32_t y_heads, const tbe_rotation_args* a) {
    return !runs_meet(runs_of(x, a, x_heads), runs_of(y, a, y_heads));
}
static bool apart_or_same(const tbe_rows& from, const tbe_rows& to, const tbe_rotation_args* a, const int32_t heads) {
    if (heads == 0) return true;
    if (from.data != to.data) return apart(from, heads, to, heads, a);
    return (a->rows <= 1 || from.row_stride == to.row_stride) && (heads == 1 || from.head_stride == to.head_stride);
}
static tbe_status rotation_call(const tbe_handle* h, const tbe_rotation_args* a, RotateCall& r) {
    const tbe_status st = check_rotation(h, a);
    if (st != TBE_OK) return st;
    if (a->norm && (a->q_weight || a->k_weight) && !io_known(a->weight_dtype)) return TBE_EDTYPE;
    const size_t w = a->norm && io_known(a->weight_dtype) ? io_size(a->weight_dtype) : 1;
    if (a->norm && (!multiple_of(a->q_weight, w) || !multiple_of(a->k_weight, w))) return TBE_EINVAL;
    if ((!a->positions && a->rows > 0) || !multiple_of(a->positions, a->index_dtype == TBE_I32 ? 4 : 8)) return TBE_EINVAL;
    if ((!a->frequencies && a->rotary_dim > 0) || !multiple_of(a->frequencies, 8)) return TBE_EINVAL;
    if (!isfinite(a->amplitude) || (a->norm && (!isfinite(a->eps) || a->eps < 0.f))) return TBE_EINVAL;
    r = RotateCall{};
    r.positions = a->positions; r.positions32 = a->index_dtype == TBE_I32;
    r.frequencies = a->frequencies;
    r.rows = a->rows; r.dim = a->head_dim; r.turned = a->rotary_dim;
    r.io = (int)a->dtype; r.param_io = (int)a->weight_dtype;
    r.pairs = a->interleaved != 0; r.norm = a->norm != 0;
    r.eps = a->eps; r.amplitude = a->amplitude;
    r.part[0].heads = a->q_heads; r.part[1].heads = a->k_heads;
    if (r.norm) {
        r.part[0].weight = a->q_weight; r.part[1].weight = a->k_weight;
    }
    return TBE_OK;
}

tbe_status tbe_rotate_heads(const tbe_handle* h, const tbe_rotation_args* args, tbe_rows q, tbe_rows k, tbe_rows q_out, tbe_rows k_out,
                            void* hip_stream) {
    RotateCall r;
    const tbe_status st = rotation_call(h, args, r);
    if (st != TBE_OK) return st;
    if (!loose_rows_ok(q, args, args->q_heads) || !loose_rows_ok(k, args, args->k_heads)) return TBE_EINVAL;
    if (!loose_result_ok(q_out, args, args->q_heads) || !loose_result_ok(k_out, args, args->k_heads)) return TBE_EINVAL;
    const int32_t nq = args->q_heads, nk = args->k_heads;
    if (!apart_or_same(q, q_out, args, nq) || !apart_or_same(k, k_out, args, nk)) return TBE_EINVAL;
    if (!apart(q_out, nq, k_out, nk, args) || !apart(q_out, nq, k, nk, args) || !apart(k_out, nk, q, nq, args)) return TBE_EINVAL;
    if (args->rows == 0) return TBE_OK;
    r.part[0].x = q; r.part[0].y = q_out;
    r.part[1].x = k; r.part[1].y = k_out;
    return done(launch_rotate(h, r, false, static_cast<hipStream_t>(hip_stream)));
}

tbe_status tbe_rotate_workspace_bytes(const tbe_handle* h, const tbe_rotation_args* args, size_t* bytes) {
    if (!bytes) return TBE_EINVAL;
    const tbe_status st = check_rotation(h, args);
    if (st == TBE_OK) *bytes = rotate_workspace(args->head_dim);
    return st;
}

tbe_status tbe_rotate_heads_backward(const tbe_handle* h, const tbe_rotation_args* args, tbe_rows dq_out, tbe_rows dk_out, tbe_rows q,
                                     tbe_rows k, tbe_rows dq, tbe_rows dk, void* dq_weight, void* dk_weight, void* workspace,
                                     size_t workspace_bytes, void* hip_stream) {
    RotateCall r;
    const tbe_status st = rotation_call(h, args, r);
    if (st != TBE_OK) return st;
    const int32_t nq = args->q_heads, nk = args->k_heads;
    if (!loose_rows_ok(dq_out, args, nq) || !loose_rows_ok(dk_out, args, nk) || !loose_result_ok(dq, args, nq) || !loose_result_ok(dk, args, nk)) return TBE_EINVAL;
    if (!apart_or_same(dq_out, dq, args, nq) || !apart_or_same(dk_out, dk, args, nk)) return TBE_EINVAL;
    if (!apart(dq, nq, dk, nk, args) || !apart(dq, nq, dk_out, nk, args) || !apart(dk, nk, dq_out, nq, args)) return TBE_EINVAL;
    if (r.norm) {
        if (!loose_rows_ok(q, args, nq) || !loose_rows_ok(k, args, nk) || !apart_or_same(q, dq, args, nq) || !apart_or_same(k, dk, args, nk)) return TBE_EINVAL;
        if (!apart(dq, nq, k, nk, args) || !apart(dk, nk, q, nq, args)) return TBE_EINVAL;
    } else if (dq_weight || dk_weight) {
        return TBE_EINVAL;
    }
    if (dq_weight || dk_weight) {
        if (!io_known(args->weight_dtype)) return TBE_EDTYPE;
        const size_t w = io_size(args->weight_dtype);
        if (!multiple_of(dq_weight, w) || !multiple_of(dk_weight, w) || !workspace || !multiple_of(workspace, 256)) return TBE_EINVAL;
        if (workspace_bytes < rotate_workspace(args->head_dim)) return TBE_EWORKSPACE;
    } else if (args->rows == 0) {
        return TBE_OK;
    }
    r.part[0].dy = dq_out; r.part[0].x = q; r.part[0].y = dq; r.part[0].dw = dq_weight;
    r.part[1].dy = dk_out; r.part[1].x = k; r.part[1].y = dk; r.part[1].dw = dk_weight;
    r.workspace = workspace;
    return done(launch_rotate(h, r, true, static_cast<hipStream_t>(hip_stream)));
}

tbe_status tbe_rotary_frequencies(int32_t rotary_dim, double base, tbe_rotary_scaling scaling, double factor, double context, double low_turns,
                                  double high_turns, double* frequencies) {
    if (rotary_dim < 2 || rotary_dim > kRotateMaxDim || rotary_dim % 2 != 0 || (scaling == TBE_ROTARY_BASE && rotary_dim < 4)) return TBE_ESHAPE;
    if (scaling < TBE_ROTARY_PLAIN || scaling > TBE_ROTARY_TURNS) return TBE_EDTYPE;
    if (!frequencies || !isfinite(base) || !(base > 1.0)) return TBE_EINVAL;
    if (scaling != TBE_ROTARY_PLAIN && !(isfinite(factor) && factor >= 1.0)) return TBE_EINVAL;
    if (scaling == TBE_ROTARY_TURNS && !(isfinite(context) && context > 0.0 && low_turns >= 0.0 && low_turns < high_turns && isfinite(high_turns))) return TBE_EINVAL;
    if (scaling == TBE_ROTARY_BASE) base *= pow(factor, (double)rotary_dim / (rotary_dim - 2));
    if (!isfinite(base)) return TBE_EINVAL;
    for (int j = 0; j < rotary_dim / 2; ++j) {
        double f = pow(base, -2.0 * j / rotary_dim);
        if (scaling == TBE_ROTARY_LINEAR) f /= factor;
        if (scaling == TBE_ROTARY_TURNS) {
            const double at = (context * f / 6.283185307179586477 - low_turns) / (high_turns - low_turns), kept = at < 0.0 ? 0.0 : (at > 1.0 ? 1.0 : at);
            f = kept * f + (1.0 - kept) * f / factor;
        }
        frequencies[j] = f;
    }
    return TBE_OK;
}

static bool code_rows(const tbe_rows& m, float* scales, const tbe_cache* c, CodeRows& v) {
    if (c->rows > 0 && (!m.data || !scales)) return false;
    if (!multiple_of(m.data, 16) || !multiple_of(scales, 4)) return false;
    if (m.row_stride < 0 || m.row_stride >= 1 << 22 || m.row_stride % 16 != 0 || m.head_stride < 0 || m.head_stride >= (int64_t)1 << 40 || m.head_stride % 16 != 0) return false;
    if ((c->rows > 1 && m.row_stride < c->head_dim) || (c->heads > 1 && m.head_stride < c->head_dim)) return false;
    v.codes.p = static_cast<const char*>(m.data); v.codes.row = m.row_stride; v.codes.head = m.head_stride;
    v.scales = scales;
    return true;
}
static tbe_status check_cache(const tbe_handle* h, const tbe_cache* c, CodeRows (&v)[2]) {
    if (!h || !c) return TBE_EINVAL;
    if (c->code != TBE_CODE_E4M3 && c->code != TBE_CODE_I8) return TBE_EDTYPE;
    if (c->rows < 0 || c->rows > ((int64_t)1 << 31) - 4096 || c->heads < 1 || c->heads > 1024) return TBE_ESHAPE;
    if (c->head_dim < 16 || c->head_dim > kAttnMaxDim || c->head_dim % 16 != 0) return TBE_ESHAPE;
    return code_rows(c->k, c->k_scales, c, v[0]) && code_rows(c->v, c->v_scales, c, v[1]) ? TBE_OK : TBE_EINVAL;
}
static tbe_status cache_copy(const tbe_handle* h, const tbe_cache* cache, const tbe_rows& k, const tbe_rows& v, const tbe_io_dtype dtype, const void* slots,
                             const tbe_index_dtype index_dtype, const int64_t rows, const bool write, void* hip_stream) {
    CacheCopyCall c{};
    const tbe_status st = check_cache(h, cache, c.cache);
    if (st != TBE_OK) return st;
    if (!io_known(dtype) || (index_dtype != TBE_I64 && index_dtype != TBE_I32)) return TBE_EDTYPE;
    if (rows < 0 || rows >= (int64_t)1 << 31) return TBE_ESHAPE;
    if (write && cache->rows > 0) {
        HeadRuns m[2];
        for (int i = 0; i < 2; ++i) {
            const RowsView& v = c.cache[i].codes;
            m[i] = HeadRuns{v.p, v.row, v.head, cache->rows, cache->heads, cache->head_dim};
            if (!runs_apart(m[i])) return TBE_EINVAL;
        }
        const int64_t bytes = 4 * cache->rows;   // of a head's scales
        const HeadRuns ks{cache->k_scales, 0, bytes, 1, cache->heads, bytes}, vs{cache->v_scales, 0, bytes, 1, cache->heads, bytes};
        if (runs_meet(m[0], m[1]) || runs_meet(ks, vs)) return TBE_EINVAL;
    }
    tbe_rotation_args as{};   // (the same kind of matrix)
    as.dtype = dtype; as.rows = rows; as.head_dim = cache->head_dim;
    if (write ? !loose_rows_ok(k, &as, cache->heads) || !loose_rows_ok(v, &as, cache->heads)
              : !loose_result_ok(k, &as, cache->heads) || !loose_result_ok(v, &as, cache->heads) || !apart(k, cache->heads, v, cache->heads, &as)) return TBE_EINVAL;
    if ((!slots && rows > 0) || !multiple_of(slots, index_dtype == TBE_I32 ? 4 : 8)) return TBE_EINVAL;
    if (rows == 0) return TBE_OK;
    c.rows_of[0] = k; c.rows_of[1] = v;
    c.slots = slots; c.slots32 = index_dtype == TBE_I32;
    c.rows = rows; c.cache_rows = cache->rows; c.heads = cache->heads; c.dim = cache->head_dim; c.io = (int)dtype; c.i8 = cache->code == TBE_CODE_I8;
    return done(launch_cache_copy(h, c, write, static_cast<hipStream_t>(hip_stream)));
}

tbe_status tbe_cache_write(const tbe_handle* h, const tbe_cache* cache, tbe_rows k, tbe_rows v, tbe_io_dtype dtype, const void* slots,
                           tbe_index_dtype index_dtype, int64_t rows, void* hip_stream) {
    return cache_copy(h, cache, k, v, dtype, slots, index_dtype, rows, true, hip_stream);
}
tbe_status tbe_cache_read(const tbe_handle* h, const tbe_cache* cache, const void* slots, tbe_index_dtype index_dtype, int64_t rows, tbe_rows k,
                          tbe_rows v, tbe_io_dtype dtype, void* hip_stream) {
    return cache_copy(h, cache, k, v, dtype, slots, index_dtype, rows, false, hip_stream);
}

tbe_status tbe_cache_attention_workspace_bytes(const tbe_handle* h, const tbe_attention_args* args, size_t* bytes) {
    if (!bytes) return TBE_EINVAL;
    const tbe_status st = check_attention_sizes(h, args);
    if (st != TBE_OK) return st;
    if (args->head_dim % 16 != 0) return TBE_ESHAPE;
    AttnShape sh = attention_shape(args);
    sh.buckets = args->buckets;
    *bytes = cache_attn_workspace(sh);
    return TBE_OK;
}

tbe_status tbe_cache_attention(const tbe_handle* h, const tbe_attention_args* args, const tbe_cache* cache, tbe_rows out, float* lse, void* workspace,
                               size_t workspace_bytes, void* hip_stream) {
    CodeRows rows[2];
    tbe_status st = check_cache(h, cache, rows);
    if (st != TBE_OK) return st;
    AttnArgs k;
    st = attention_args(h, args, k, false);
    if (st != TBE_OK) return st;
    if (args->kv_heads != cache->heads || args->head_dim != cache->head_dim || args->k_rows != cache->rows) return TBE_ESHAPE;
    if (!rows_view(out, args->q_rows, args->heads, args, true, k.o) || !multiple_of(lse, 4)) return TBE_EINVAL;
    k.lse = lse;
    const AttnShape sh = attention_shape(args);
    const CacheAttnPlan p = cache_attn_plan(sh, args->dtype == TBE_IO_BF16 && cache->code == TBE_CODE_E4M3);
    const size_t need = p.spans + p.part_ml + p.part_o;
    if (need > 0) {
        if (!workspace || !multiple_of(workspace, 256)) return TBE_EINVAL;
        if (workspace_bytes < need) return TBE_EWORKSPACE;
    }
    if (!cache_attn_grid_ok(sh, p)) return TBE_ESHAPE;
    if (args->q_rows == 0) return TBE_OK;
    return done(launch_cache_attention(h, k, rows, cache->code == TBE_CODE_I8, p, (int)args->dtype, workspace, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
