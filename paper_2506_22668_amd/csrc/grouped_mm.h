// What the two forms of the products by group share (no part of the ABI).
#pragma once
#include "feature_ops.h"
#include "group_range.h"
#include "grouped_forms.h"

struct MmArgs {
  int rows, inner, outer, groups;
  const void *w, *x, *dy, *gate;
  int64_t xs, dys, gs, ys;
  const int64_t* offsets;
  const int32_t* order;
  const float* bias;
  int relu, col_tiles;
  void* y;            // the product by rows (y, or dx)
  void* dw;
  float* db;
  // x held in 8 bits (xs: the distance of its rows of codes; the gate is codes too)
  const uint8_t *codes, *scales;
  int64_t scales_stride;
};

// tiles of 2^shift rows that the groups and the rows of none can have: every group may end inside one
static inline int64_t ds_most_tiles(const MmArgs& a, int shift) {
  return ds_most_parts(a.rows, 1 << shift, a.groups + 1);
}

// The product by rows in tiles through LDS (grouped_tiles.hip); transposed: dx = dy w^T
int ds_launch_row_tiles(ds_ctx* ctx, int dtype, bool transposed, MmArgs& a);
// The gradient of the weights in tiles; partial: ds_weight_tiles_bytes of scratch
int64_t ds_weight_tiles_bytes(int dtype, int rows, int inner, int outer);
int ds_launch_weight_tiles(ds_ctx* ctx, int dtype, MmArgs& a, void* partial);
// The same where x, and the gate, are held in 8 bits (packed_tiles.hip)
int ds_launch_row_tiles_packed(ds_ctx* ctx, int dtype, MmArgs& a);
int ds_launch_weight_tiles_packed(ds_ctx* ctx, int dtype, MmArgs& a, void* partial);
