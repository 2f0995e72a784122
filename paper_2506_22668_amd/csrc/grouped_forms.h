// Which form of the products by group a call takes. Host functions of its sizes alone (tests/test_grouped_forms.py compiles them by themselves).
//
// Each form has a price in us on 256 compute units, from the number of its workgroups, how many run at a time, and what one takes for its share of the
// contraction; the sizes of groups are not known on the host, so all are taken to be of the mean size. What that costs where they are not, both gradients
// in bf16 by 256 x 256, rows spread evenly / all in one group: 65,536 rows, 1,024 groups 151 / 575 us; 4,096 rows, 256 groups 37 / 357 us.
//
// Measured, each form forced, at 323 shapes (1, 8 and 64 equal groups of 8 to 16,000 rows, eight pairs of widths of 64 to 4,096, 513 x 300 among them, bf16 and
// fp32; profiles/operators_forms.md): forward the choice is 0.8 % off the faster form on average and more than 12 % at 3 shapes, both gradients 2.5 % and 19,
// 16 of which are 513 x 300, where tiles cost more than is priced: odd rows come to them through registers. Forward in us, few / tiles:
//   8 groups by 1,024 x 1,024, bf16: 8 rows each 9 / 21, 400 28 / 23, 1,000 54 / 31; 64 groups of 200 rows by 256 x 256 23 / 11, by 64 x 64 10 / 9
#pragma once
#include <math.h>
#include <stdint.h>

#include "../../include/distshap.h"

struct ds_mm_sizes {
  int rows, inner, outer, groups;
};

constexpr double kFormUnits = 256;
constexpr double kNarrowTiles = 512;   // 16 bits: up to so many row tiles are of 128 by 128, if that many are needed (ds_narrow_tiles)

inline double ds_ceil_div(double a, double b) { return ceil(a / b); }

// fp32: 256 rows to a tile where there are about as many tiles as compute units (65,536 rows by 512 x 512: 0.36 -> 0.34 ms; with half as many tiles,
// 4,096 rows by 2,048 x 512: 0.16 -> 0.27 ms)
inline bool ds_wide_tiles(int rows, int width) { return (int64_t)(rows / 256) * ((width + 127) / 128) >= 224; }

// 16 bits: tiles of 128 by 128, of which a compute unit has two at a time, where there are no more than that: 256 by 256 would leave units idle
// (8,192 rows in 8 groups by 512 x 512: 24 us in large, 17 in small; by 1,024 x 1,024: 39, 34). With more, the large ones' fewer loads from L2
// count (131,072 rows by 512 x 512: 108, 144; by 1,024 x 1,024: 416, 520).
inline double ds_narrow_tiles(int rows, int groups, int width) {
  const double mean = ceil((double)rows / groups);
  return groups * ceil(mean / 128) * ceil(width / 128.0);
}

// Chunks of the line of steps: as many as fill the compute units with every tile once, or twice where that leaves fewer of them idle in the last
// round, but none of less than two steps (128 rows of 16 bits).
inline int ds_weight_chunks(int rows, int64_t tiles, int unit) {
  const int64_t units = (int64_t)kFormUnits;
  const auto idle = [&](int64_t p) { return (double)((p * tiles + units - 1) / units * units) / (double)(p * tiles); };
  const int64_t once = units / tiles > 1 ? units / tiles : 1, twice = 2 * units / tiles > 1 ? 2 * units / tiles : 1;
  const int64_t p = idle(twice) < 0.93 * idle(once) ? twice : once, most = rows / (2 * unit);
  return (int)(p < most ? p : most > 1 ? most : 1);
}

// the product by rows, `depth` long and `width` wide
inline bool ds_rows_in_tiles(const ds_mm_sizes& p, int dtype, int depth, int width) {
  if (p.inner < 8 || p.outer < 8) return false;   // (the tiles' loads need rows of 16 bytes at the least)
  const bool f32 = dtype == DS_ELEM_F32;
  const double mean = ds_ceil_div(p.rows, p.groups);
  const double block = mean <= 16 ? 16 : mean <= 32 ? 32 : 64;
  const double few = p.groups * ds_ceil_div(mean, block) * ds_ceil_div(width, f32 ? 64 : 128) / kFormUnits;
  const double few_us = (few > 1 ? few : 1) * (5 + (f32 ? 0.02 : 0.009) * depth);
  const double narrow = ds_narrow_tiles(p.rows, p.groups, width);
  if (!f32 && narrow <= kNarrowTiles) return 1 + (narrow > kFormUnits ? 0.026 : 0.017) * depth < few_us;
  if (!f32) return ds_ceil_div(p.groups * ds_ceil_div(mean, 256) * ds_ceil_div(width, 256), kFormUnits) * (4 + 0.025 * depth) < few_us;
  const bool wide = ds_wide_tiles(p.rows, width);
  const double rounds = ds_ceil_div(p.groups * ds_ceil_div(mean, wide ? 256 : 128) * ds_ceil_div(width, 128), kFormUnits);
  return rounds * (wide ? 13 + 0.14 * depth : 8 + 0.075 * depth) + 6 < few_us;
}

// Up to 32 rows to a group a wave of the few-rows form has columns of its own, a quarter as many, beyond that the waves of a workgroup share the
// rows (both gradients, 8 groups by 1,024 x 1,024, alone / shared: 8 rows each bf16 25 / 40 us, fp32 32 / 44; 32 rows: 28 / 42, 41 / 47; 64 rows:
// 36 / 46, 66 / 58; 128 rows: 44 / 48, 92 / 76)
inline bool ds_weights_shared(const ds_mm_sizes& p) { return (int64_t)p.rows > 32 * (int64_t)p.groups; }

inline bool ds_weights_in_tiles(const ds_mm_sizes& p, int dtype) {
  if (p.inner < 8 || p.outer < 8) return false;   // (as above, and long groups pay for it: both gradients, 100,000 rows in 3 groups, bf16, by 256 x 5 900 us, by 256 x 8 63)
  const bool f32 = dtype == DS_ELEM_F32;
  const double mean = ds_ceil_div(p.rows, p.groups), n = f32 ? 4 : 8;
  const double few = p.groups * ds_ceil_div(p.outer, 16 * n) * ds_ceil_div(p.inner, 8 * n) / kFormUnits;
  const double alone = p.groups * ds_ceil_div(p.outer, 16 * n) * ds_ceil_div(p.inner, 4 * n) / (kFormUnits * (f32 ? 16 : 8));   // (waves at a time)
  const double few_us = ds_weights_shared(p) ? (few > 1 ? few : 1) * ((f32 ? 3 : 5) + 2 * ds_ceil_div(mean, 16 * n))
                                             : (alone > 1 ? alone : 1) * (6 + 2 * ds_ceil_div(mean, 4 * n));
  const double side = f32 ? 128 : 256, unit = f32 ? 32 : 64;
  const double tiles = ds_ceil_div(p.inner, side) * ds_ceil_div(p.outer, side), chunks = ds_weight_chunks(p.rows, (int64_t)tiles, (int)unit);
  const double steps = ds_ceil_div(p.groups * ds_ceil_div(mean, unit), chunks), cut = 1 + (p.groups > chunks ? p.groups / chunks : 0) + (chunks > 1 ? 1 : 0);
  const double rounds = chunks * tiles / kFormUnits;
  const bool odd = p.inner % 4 || p.outer % 4;   // (fp32 rows that are not aligned: both gradients of 64 groups of 1,000 rows by 513 x 300, dW in few 749 us, in tiles 831)
  return (rounds > 1 ? rounds : 1) * (steps * (f32 ? odd ? 5.0 : 1.5 : 2.0) + cut * (f32 ? 8 : 5)) + (f32 ? 12 : 4) < few_us;
}

// ---- within the few-rows form -----------------------------------------------------------------------------------------------------

// Twice the waves to a workgroup that takes up to 32 rows, where workgroups are few and the contraction is long (8 rows to a group, bf16 / fp32; 8 groups by
// 4,096 x 1,024, 64 / 128 workgroups: 26.6 -> 19.7 us / 42 -> 33; 1 group by 1,024 x 1,024: 9.9 -> 11.8 / 12.1 -> 10.9; 8 groups by 1,024 x 4,096, 256 / 512
// workgroups: 15.2 -> 15.0 / 23.6 -> 25.5; 64 rows to a group: no faster anywhere)
inline bool ds_eight_waves(double workgroups, int depth, int step) { return workgroups <= 128 && depth >= 16 * step; }

// The product with W^T of half the columns to a workgroup, where those of all would be at most 128 workgroups; with more, reading the rows twice as often
// counts (both gradients in us, all / half columns; 8 groups by 1,024 x 4,096, 64 workgroups, bf16: 8 rows 73 / 59, 64 rows 80 / 65; 128 rows, 128 workgroups
// 85 / 71; 256 rows, 256 workgroups 95 / 112; fp32, 4 groups by 1,024 x 4,096: 8 rows, 64 workgroups 68 / 55, 256 rows, 256 workgroups 211 / 227)
inline bool ds_half_columns(double workgroups) { return workgroups <= 128; }

struct ds_few_form {
  int shift, cols;          // a workgroup takes 2^shift rows and so many columns
  bool half, eight_waves;   // half of the columns; eight waves, not four
};
// the product by rows, transposed: dx = dy W^T; tiny: an operand has less than 16 bytes
inline ds_few_form ds_choose_few(const ds_mm_sizes& p, int dtype, bool transposed, bool tiny) {
  const int n = dtype == DS_ELEM_F32 ? 4 : 8, depth = transposed ? p.outer : p.inner, width = transposed ? p.inner : p.outer;
  const double mean = ds_ceil_div(p.rows, p.groups);
  ds_few_form f;
  f.shift = tiny || mean > 32 ? 6 : mean > 16 ? 5 : 4;
  const double blocks = p.groups * ds_ceil_div(mean, 1 << f.shift);
  f.half = transposed && !tiny && ds_half_columns(blocks * ds_ceil_div(width, 16 * n));
  f.cols = f.half ? 8 * n : 16 * n;
  f.eight_waves = !tiny && f.shift < 6 && ds_eight_waves(blocks * ds_ceil_div(width, f.cols), depth, 4 * 4 * n);
  return f;
}
