// C ABI of the operators on sequences of looked-up rows: argument checks, workspaces.  Nothing is launched when a check fails.
#include <math.h>

#include "tbe_internal.h"

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

}  // extern "C"
