// Gradients of the products by group, in tiles, from rows that are held in 8 bits (grouped_tiles.h has the kernels).
#include "grouped_tiles.h"

int ds_launch_row_tiles_packed(ds_ctx* ctx, int dtype, MmArgs& a) {
  if (dtype == DS_ELEM_F32) return launch_rows<float, true, true>(ctx, a);
  if (dtype == DS_ELEM_BF16) return launch_rows<__bf16, true, true>(ctx, a);
  return launch_rows<_Float16, true, true>(ctx, a);
}

int ds_launch_weight_tiles_packed(ds_ctx* ctx, int dtype, MmArgs& a, void* partial) { return launch_weights_of<true>(ctx, dtype, a, (float*)partial); }
