// The rows of a group from the offsets that a caller gives. For host and device.
#pragma once
#include <stdint.h>
#ifdef __HIPCC__
#define DS_GROUP_FN __host__ __device__ inline
#else
#define DS_GROUP_FN inline
#endif

// Positions [*begin, *end) of group g in the order; g == groups: the rows of no group, behind the last group's. The offsets are the
// caller's and live on the GPU, where no host check reaches: whatever they hold, 0 <= *begin <= *end <= rows.
DS_GROUP_FN void ds_group_range(const int64_t* offsets, int groups, int rows, int g, int* begin, int* end) {
  const int64_t b = offsets[g], e = g < groups ? offsets[g + 1] : (int64_t)rows;
  *begin = b < 0 ? 0 : b > rows ? rows : (int)b;
  *end = e < *begin ? *begin : e > rows ? rows : (int)e;
}

// The row at position `at` of the order (null: the rows are sorted by group already); -1 where the order names none.
DS_GROUP_FN int ds_ordered_row(const int32_t* order, int rows, int at) {
  if (!order) return at;
  const int r = order[at];
  return r >= 0 && r < rows ? r : -1;
}
