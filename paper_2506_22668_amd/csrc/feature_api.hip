// C ABI entry points of the operators on rows of features: argument checks, then the launch.
#include <math.h>

#include "feature_ops.h"

namespace {

constexpr int kMostCols = 1 << 20, kMostNormCols = 4096, kMostGroups = 1024;
constexpr int64_t kMostRows = 1ll << 40, kMostOrdered = 1ll << 30;

bool known(int dtype) { return dtype == DS_ELEM_F32 || dtype == DS_ELEM_BF16 || dtype == DS_ELEM_F16; }
size_t element_bytes(int dtype) { return dtype == DS_ELEM_F32 ? 4 : 2; }

// a matrix argument: there where it has rows, aligned to its elements, rows of an output apart from each other
int check_rows(ds_ctx* ctx, const char* name, const void* p, int64_t stride, int64_t rows, int64_t cols, int dtype, bool out) {
  if (rows == 0) return DS_OK;
  if (!p) return ds_fail(ctx, DS_EINVAL, "%s is null", name);
  if ((uintptr_t)p % element_bytes(dtype)) return ds_fail(ctx, DS_EINVAL, "%s is not aligned to its elements", name);
  if (stride < 0 || (out && rows > 1 && stride < cols))
    return ds_fail(ctx, DS_EINVAL, "%s: rows of %lld columns cannot lie %lld apart", name, (long long)cols, (long long)stride);
  if (stride > (1ll << 40)) return ds_fail(ctx, DS_EINVAL, "%s: rows lie too far apart", name);
  return DS_OK;
}

int check_shape(ds_ctx* ctx, int dtype, int64_t rows, int64_t most_rows, int64_t cols, int64_t most_cols) {
  if (!known(dtype)) return ds_fail(ctx, DS_EINVAL, "unknown element type %d", dtype);
  if (rows < 0 || rows > most_rows) return ds_fail(ctx, DS_EINVAL, "%lld rows out of range [0, %lld]", (long long)rows, (long long)most_rows);
  if (cols < 1 || cols > most_cols) return ds_fail(ctx, DS_EINVAL, "%lld columns out of range [1, %lld]", (long long)cols, (long long)most_cols);
  return DS_OK;
}

int check_workspace(ds_ctx* ctx, const void* workspace, int64_t bytes, int64_t need) {
  if (need > 0 && (!workspace || bytes < need))
    return ds_fail(ctx, DS_ECAPACITY, "the workspace has %lld bytes, the call needs %lld", (long long)(workspace ? bytes : 0), (long long)need);
  if (need > 0 && (uintptr_t)workspace % 16) return ds_fail(ctx, DS_EINVAL, "the workspace is not aligned to 16 bytes");
  return DS_OK;
}

int check_groups(ds_ctx* ctx, int64_t groups, const int64_t* offsets) {
  if (groups < 1 || groups > kMostGroups) return ds_fail(ctx, DS_EINVAL, "%lld groups out of range [1, %d]", (long long)groups, kMostGroups);
  if (!offsets) return ds_fail(ctx, DS_EINVAL, "offsets is null");
  return DS_OK;
}

int64_t norm_bytes(int64_t rows, int64_t cols) { return ds_layer_norm_partials(rows, (int)cols) * 2 * cols * (int64_t)sizeof(float); }
int64_t group_bytes(int64_t rows, int64_t groups) {
  const int64_t blocks = ds_group_blocks((int)rows);
  return blocks > 1 ? (blocks + 1) * (groups + 1) * (int64_t)sizeof(int32_t) : 0;
}

}  // namespace

extern "C" {

int ds_layer_norm(ds_ctx* ctx, int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const float* weight,
                  const float* bias, float eps, void* y, int64_t y_stride, float* mean, float* rstd) {
  if (!ctx) return DS_EINVAL;
  DS_TRY(check_shape(ctx, dtype, rows, kMostRows, cols, kMostNormCols));
  if (!(eps >= 0.f) || isinf(eps)) return ds_fail(ctx, DS_EINVAL, "eps must be a finite number, not below 0");
  DS_TRY(check_rows(ctx, "x", x, x_stride, rows, cols, dtype, false));
  DS_TRY(check_rows(ctx, "y", y, y_stride, rows, cols, dtype, true));
  DS_HIP(ctx, hipSetDevice(ctx->device));
  return ds_launch_layer_norm(ctx, dtype, rows, (int)cols, {x, x_stride}, weight, bias, eps, {y, y_stride}, mean, rstd);
}

int ds_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* bytes) {
  if (!bytes || rows < 0 || rows > kMostRows || cols < 1 || cols > kMostNormCols) return DS_EINVAL;
  *bytes = norm_bytes(rows, cols);
  return DS_OK;
}

int ds_layer_norm_backward(ds_ctx* ctx, int32_t dtype, int64_t rows, int64_t cols, const void* dy, int64_t dy_stride, const void* x,
                           int64_t x_stride, const float* mean, const float* rstd, const float* weight, void* dx,
                           int64_t dx_stride, float* dweight, float* dbias, void* workspace, int64_t workspace_bytes) {
  if (!ctx) return DS_EINVAL;
  DS_TRY(check_shape(ctx, dtype, rows, kMostRows, cols, kMostNormCols));
  DS_TRY(check_rows(ctx, "dy", dy, dy_stride, rows, cols, dtype, false));
  DS_TRY(check_rows(ctx, "x", x, x_stride, rows, cols, dtype, false));
  DS_TRY(check_rows(ctx, "dx", dx, dx_stride, rows, cols, dtype, true));
  if (rows > 0 && (!mean || !rstd)) return ds_fail(ctx, DS_EINVAL, "mean and rstd of the forward pass are needed");
  if (!dweight || !dbias) return ds_fail(ctx, DS_EINVAL, "dweight and dbias are needed");
  DS_TRY(check_workspace(ctx, workspace, workspace_bytes, norm_bytes(rows, cols)));
  DS_HIP(ctx, hipSetDevice(ctx->device));
  return ds_launch_layer_norm_backward(ctx, dtype, rows, (int)cols, {dy, dy_stride}, {x, x_stride}, mean, rstd, weight,
                                       {dx, dx_stride}, dweight, dbias, (float*)workspace);
}

int ds_dropout(ds_ctx* ctx, int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* residual,
               int64_t residual_stride, double p, uint64_t seed, uint32_t tag, void* y, int64_t y_stride) {
  if (!ctx) return DS_EINVAL;
  DS_TRY(check_shape(ctx, dtype, rows, kMostRows, cols, kMostCols));
  if (!(p >= 0.0 && p <= 1.0)) return ds_fail(ctx, DS_EINVAL, "the share that is dropped must lie in [0, 1]");
  DS_TRY(check_rows(ctx, "x", x, x_stride, rows, cols, dtype, false));
  if (residual) DS_TRY(check_rows(ctx, "residual", residual, residual_stride, rows, cols, dtype, false));
  DS_TRY(check_rows(ctx, "y", y, y_stride, rows, cols, dtype, true));
  DS_HIP(ctx, hipSetDevice(ctx->device));
  return ds_launch_dropout(ctx, dtype, rows, (int)cols, {x, x_stride}, {residual, residual_stride}, (int)nearbyint(p * 65536.0), seed,
                           tag, {y, y_stride});
}

int ds_group_rows_workspace(int64_t rows, int64_t groups, int64_t* bytes) {
  if (!bytes || rows < 0 || rows > kMostOrdered || groups < 1 || groups > kMostGroups) return DS_EINVAL;
  *bytes = group_bytes(rows, groups);
  return DS_OK;
}

int ds_group_rows(ds_ctx* ctx, const int32_t* ids, int64_t rows, int64_t groups, int64_t* offsets, int32_t* order, void* workspace,
                  int64_t workspace_bytes) {
  if (!ctx) return DS_EINVAL;
  if (rows < 0 || rows > kMostOrdered) return ds_fail(ctx, DS_EINVAL, "%lld rows out of range [0, %lld]", (long long)rows, (long long)kMostOrdered);
  DS_TRY(check_groups(ctx, groups, offsets));
  if (rows > 0 && (!ids || !order)) return ds_fail(ctx, DS_EINVAL, "%s is null", ids ? "order" : "ids");
  DS_TRY(check_workspace(ctx, workspace, workspace_bytes, group_bytes(rows, groups)));
  DS_HIP(ctx, hipSetDevice(ctx->device));
  return ds_launch_group_rows(ctx, ids, (int)rows, (int)groups, offsets, order, (int32_t*)workspace);
}

int ds_grouped_mm(ds_ctx* ctx, int32_t dtype, int64_t rows, int64_t inner, int64_t outer, int64_t groups, const void* x,
                  int64_t x_stride, const void* w, const int64_t* offsets, const int32_t* order, const float* bias, int32_t relu,
                  void* y, int64_t y_stride) {
  if (!ctx) return DS_EINVAL;
  DS_TRY(check_shape(ctx, dtype, rows, kMostOrdered, inner, kMostCols));
  DS_TRY(check_shape(ctx, dtype, rows, kMostOrdered, outer, kMostCols));
  DS_TRY(check_groups(ctx, groups, offsets));
  DS_TRY(check_rows(ctx, "x", x, x_stride, rows, inner, dtype, false));
  DS_TRY(check_rows(ctx, "w", w, outer, groups, outer, dtype, false));
  DS_TRY(check_rows(ctx, "y", y, y_stride, rows, outer, dtype, true));
  DS_HIP(ctx, hipSetDevice(ctx->device));
  const ds_grouped p = {(int)rows, (int)inner, (int)outer, (int)groups, w, offsets, order};
  return ds_launch_grouped_mm(ctx, dtype, p, {x, x_stride}, bias, relu != 0, {y, y_stride});
}

int ds_grouped_mm_backward_workspace(int32_t dtype, int64_t rows, int64_t inner, int64_t outer, int64_t groups, int64_t* bytes) {
  if (!bytes || !known(dtype) || rows < 0 || rows > kMostOrdered || inner < 1 || inner > kMostCols || outer < 1 || outer > kMostCols ||
      groups < 1 || groups > kMostGroups)
    return DS_EINVAL;
  *bytes = ds_grouped_mm_backward_bytes(dtype, {(int)rows, (int)inner, (int)outer, (int)groups, nullptr, nullptr, nullptr});
  return DS_OK;
}

int ds_grouped_mm_backward(ds_ctx* ctx, int32_t dtype, int64_t rows, int64_t inner, int64_t outer, int64_t groups, const void* dy,
                           int64_t dy_stride, const void* x, int64_t x_stride, const void* w, const int64_t* offsets,
                           const int32_t* order, const void* gate, int64_t gate_stride, void* dx, int64_t dx_stride, void* dw,
                           float* db, void* workspace, int64_t workspace_bytes) {
  if (!ctx) return DS_EINVAL;
  DS_TRY(check_shape(ctx, dtype, rows, kMostOrdered, inner, kMostCols));
  DS_TRY(check_shape(ctx, dtype, rows, kMostOrdered, outer, kMostCols));
  DS_TRY(check_groups(ctx, groups, offsets));
  DS_TRY(check_rows(ctx, "dy", dy, dy_stride, rows, outer, dtype, false));
  DS_TRY(check_rows(ctx, "x", x, x_stride, rows, inner, dtype, false));
  DS_TRY(check_rows(ctx, "w", w, outer, groups, outer, dtype, false));
  if (gate) DS_TRY(check_rows(ctx, "gate", gate, gate_stride, rows, inner, dtype, false));
  DS_TRY(check_rows(ctx, "dx", dx, dx_stride, rows, inner, dtype, true));
  DS_TRY(check_rows(ctx, "dw", dw, outer, groups, outer, dtype, true));
  if (!db) return ds_fail(ctx, DS_EINVAL, "db is null");
  const ds_grouped p = {(int)rows, (int)inner, (int)outer, (int)groups, w, offsets, order};
  DS_TRY(check_workspace(ctx, workspace, workspace_bytes, ds_grouped_mm_backward_bytes(dtype, p)));
  DS_HIP(ctx, hipSetDevice(ctx->device));
  return ds_launch_grouped_mm_backward(ctx, dtype, p, {dy, dy_stride}, {x, x_stride}, {gate, gate_stride}, {dx, dx_stride}, dw, db,
                                       workspace);
}

}  // extern "C"
