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

// The rows cut into tiles (or steps) of `size`, group by group; `parts` counts the groups that can end inside one, the rows of no group among
// them where they have tiles. As many as there can be if the offsets ascend: at most rows / 16 + 1,025.
DS_GROUP_FN int ds_most_parts(int rows, int size, int parts) { return rows / size + (parts < rows ? parts : rows); }
DS_GROUP_FN int ds_parts_of(int begin, int end, int size) { return (int)(((int64_t)(end - begin) + size - 1) / size); }

// Sums of tiles stop at `most`. Offsets that do not ascend can give every group all rows, and 1,024 times 2^30 rows are more tiles than an int
// counts. Sums of offsets that ascend never meet the end, and a capped sum is associative, so it can be formed in any order.
DS_GROUP_FN int ds_add_parts(int a, int b, int most) { return a + b < most ? a + b : most; }

// Workgroups [*first, *last] of `wgs` that share the `own` (> 0) steps of a group, in a line of `all` steps cut evenly, where `before` steps lie in
// front of them (capped sums both). owner(x): the workgroup of step x.
template <typename Owner>
DS_GROUP_FN void ds_group_owners(int before, int own, int all, const Owner& owner, int* first, int* last) {
  *first = owner(before < all ? before : all - 1);
  *last = owner(ds_add_parts(before, own, all) - 1);
}

// A launch counts its threads in 32 bits a dimension; of one with more, HIP leaves workgroups out without an error.
inline int64_t ds_most_workgroups(int threads) { return 0xffffffffll / threads; }
struct ds_lines {
  unsigned x, y;   // workgroup number blockIdx.y * x + blockIdx.x; up to y - 1 of them are too many
};
inline ds_lines ds_launch_lines(int64_t workgroups, int threads) {
  const int64_t most = ds_most_workgroups(threads), y = (workgroups + most - 1) / most, x = (workgroups + y - 1) / y;
  return {(unsigned)x, (unsigned)y};
}
