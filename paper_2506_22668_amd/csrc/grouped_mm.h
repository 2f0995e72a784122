// What the two forms of the products by group share (no part of the ABI).
#pragma once
#include "feature_ops.h"
#include "group_range.h"

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
// what the choice between the forms has to know of the tiles
bool ds_wide_tiles(int rows, int width);                           // fp32: 256 rows to a tile
constexpr double kNarrowTiles = 512;                               // 16 bits: up to so many tiles are of 128 by 128 ..
double ds_narrow_tiles(int rows, int groups, int width);           // .. if this many are needed
int ds_weight_chunks(int rows, int64_t tiles, int unit);           // stretches that the rows are cut into, in units of `unit` rows
