// Products of rows with the weights of their group where a group has many rows: launches (grouped_tiles.h has the kernels).
#include "grouped_tiles.h"

int ds_launch_row_tiles(ds_ctx* ctx, int dtype, bool transposed, MmArgs& a) {
  if (dtype == DS_ELEM_F32) return transposed ? launch_rows<float, true, false>(ctx, a) : launch_rows<float, false, false>(ctx, a);
  if (dtype == DS_ELEM_BF16) return transposed ? launch_rows<__bf16, true, false>(ctx, a) : launch_rows<__bf16, false, false>(ctx, a);
  return transposed ? launch_rows<_Float16, true, false>(ctx, a) : launch_rows<_Float16, false, false>(ctx, a);
}

int64_t ds_weight_tiles_bytes(int dtype, int rows, int inner, int outer) {
  const int64_t side = dtype == DS_ELEM_F32 ? 128 : 256;
  const int64_t tiles = dtype == DS_ELEM_F32 ? weight_tiles<float, 128, 128>(inner, outer) : weight_tiles<__bf16, 256, 256>(inner, outer);
  const int64_t chunks = ds_weight_chunks(rows, tiles, dtype == DS_ELEM_F32 ? 32 : 64);
  return chunks > 1 ? tiles * chunks * 2 * (side * side + side) * (int64_t)sizeof(float) : 0;
}

int ds_launch_weight_tiles(ds_ctx* ctx, int dtype, MmArgs& a, void* partial) { return launch_weights_of<false>(ctx, dtype, a, (float*)partial); }
