// Launchers of the operators on rows of features (no part of the ABI); arguments are checked in feature_api.hip.
#pragma once
#include "internal.h"

struct ds_rows {          // a matrix whose rows lie `stride` elements apart
  const void* data;
  int64_t stride;
};

int ds_launch_layer_norm(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows x, const float* weight, const float* bias,
                         float eps, ds_rows y, float* mean, float* rstd);
int64_t ds_layer_norm_partials(int64_t rows, int cols);   // pairs of partial rows that the backward pass leaves
int ds_launch_layer_norm_backward(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows dy, ds_rows x, const float* mean,
                                  const float* rstd, const float* weight, ds_rows dx, float* dweight, float* dbias,
                                  float* partial);
int ds_launch_dropout(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows x, ds_rows residual, int threshold, uint64_t seed,
                      uint32_t tag, ds_rows y);
int ds_group_blocks(int rows);
int ds_launch_group_rows(ds_ctx* ctx, const int32_t* ids, int rows, int groups, int64_t* offsets, int32_t* order, int32_t* counts);

struct ds_grouped {
  int rows, inner, outer, groups;
  const void* w;            // [groups x inner x outer]
  const int64_t* offsets;   // [groups + 1]
  const int32_t* order;     // [rows] or null
};
int ds_launch_grouped_mm(ds_ctx* ctx, int dtype, const ds_grouped& p, ds_rows x, const float* bias, int relu, ds_rows y);
int64_t ds_grouped_mm_backward_bytes(int dtype, const ds_grouped& p);
int ds_launch_grouped_mm_backward(ds_ctx* ctx, int dtype, const ds_grouped& p, ds_rows dy, ds_rows x, ds_rows gate, ds_rows dx,
                                  void* dw, float* db, void* workspace);
