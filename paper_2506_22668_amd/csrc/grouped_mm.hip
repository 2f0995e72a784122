// Products of rows with the weights of their group, and their gradients.
//
//   forward:   y[r] = x[r] W_g + b_g (ReLU)              for the rows r of group g, zeros for the rows of no group
//   backward:  dx[r] = (gate[r] > 0) dy[r] W_g^T,  dW_g = sum_r x[r]^T dy[r],  db_g = sum_r dy[r]
//
// The rows of group g are those at positions offsets[g] .. offsets[g + 1] of `order`. Sizes of groups are known on the GPU
// alone: the grid has a tile for every one that there can be, and a workgroup finds its rows from the offsets.
// All products go through the matrix cores, fp32 ones on their fp32 form, and are summed in fp32.
#include <type_traits>

#include "grouped_mm.h"
#include "rows.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// d += a b on 16 x 16 with a lane's piece of both operands: lane l gives row (column) l % 16 and the contraction's indices
// N (l / 16) .. + N - 1; d: column l % 16, rows 4 (l / 16) .. + 3.
__device__ __forceinline__ f32x4 multiply(PieceV<__bf16> a, PieceV<__bf16> b, f32x4 d) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(PieceV<_Float16> a, PieceV<_Float16> b, f32x4 d) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(PieceV<float> a, PieceV<float> b, f32x4 d) {
#pragma unroll
  for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], d, 0, 0, 0);
  return d;
}

constexpr int kWaves = 4;   // of a workgroup: they share the contraction

// ---- few rows to a group --------------------------------------------------------------------------------------------------
// A workgroup takes 16 RB rows of one group and 16 N columns (N = elements of a 16-byte piece), each of its waves every
// fourth step of the contraction; their sums meet in LDS. No operand is shared between waves, so none goes through LDS: a
// wave has eight pieces of W a step in flight without a barrier. W is read in its own order: where its rows run along the
// columns of the result (TRANSPOSED false: N steps of the contraction by 8 columns to a lane) the lane turns its square of
// elements around in registers; column j of the squares of 16 lanes is an operand, so that a lane ends up with N neighbouring columns of a
// row. TRANSPOSED: the product with W^T, whose pieces are operands as they are (HALF: of half
// the columns and twice the contraction: more workgroups, and a wave reads whole lines of 128 bytes of a row; see ds_half_columns).
// Loads have no branches, which they would be waited for at: a piece that reaches over its row's end brings the next row's elements along. Columns
// that there are not lead to results that nobody stores; where the contraction ends, the last step clears them. A piece that would reach over
// the matrix' end, which it can in its last N rows alone, is read so that it ends there, and shifted. (TINY: matrices of less than 16 bytes, element by element.)
// Bound by reading W, from memory once if a group has one tile of rows: 8 rows in 8 groups by 1,024 x 4,096 bf16 14.1 us, 4.8 TB/s. (64 rows of 16 bits
// to a workgroup take 130 + 128 registers, dx 136 + 128 or 196 + 68: one wave to a SIMD.)
template <typename T, int RB, int WAVES, bool TRANSPOSED, bool HALF, bool TINY>
__global__ __launch_bounds__(64 * WAVES) void few_rows_kernel(MmArgs a) {
  constexpr int N = Piece<T>::N, SHIFT = RB == 1 ? 4 : RB == 2 ? 5 : 6;
  constexpr int COLS = HALF ? N / 2 : N, HALVES = N / COLS, STEP = WAVES * 4 * N * HALVES;   // of a lane's columns, and pieces of each
  __shared__ float meet[WAVES][4][64][COLS];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int at = (int)(blockIdx.y * gridDim.x + blockIdx.x);   // (see ds_launch_lines)
  const int tile = at / a.col_tiles, width = TRANSPOSED ? a.inner : a.outer, depth = TRANSPOSED ? a.outer : a.inner;
  const int col = (at % a.col_tiles) * 16 * COLS;
  GroupTiles all(a.offsets, a.groups, a.rows, SHIFT);
  if (tile >= all.count()) return;
  const GroupTile gt = all.find(tile);
  int row[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) row[r] = gt.begin + 16 * r + m < gt.end ? ds_ordered_row(a.order, a.rows, gt.begin + 16 * r + m) : -1;
  f32x4 acc[RB][COLS] = {};
  const int64_t xs = TRANSPOSED ? a.dys : a.xs;
  const T* x = (const T*)(TRANSPOSED ? a.dy : a.x);
  if (gt.group < a.groups) {
    const T *w = (const T*)a.w + (int64_t)gt.group * a.inner * a.outer, *w_end = (const T*)a.w + (int64_t)a.groups * a.inner * a.outer;
    const T* x_end = x + (int64_t)(a.rows - 1) * xs + depth;
    const int n0 = col + COLS * m;   // the lane's columns
    PieceV<T> wp[N], xp[RB * HALVES];
    const auto over = [](const T* p, const T* end) -> unsigned {
      const int64_t by = p + N - end;
      return by <= 0 ? 0 : by < N ? (unsigned)by : N;
    };
    const auto w_at = [&](int k, int i) -> const T* {
      if constexpr (TRANSPOSED) return w + (int64_t)min(n0 + i / HALVES, width - 1) * a.outer + min(k + i % HALVES * 4 * N, depth - 1);
      else return w + (int64_t)min(k + i, depth - 1) * a.outer + min(n0, width - 1);
    };
    const auto x_at = [&](int k, int i) -> const T* {
      const int r = row[i / HALVES];
      return x + (r < 0 ? 0 : r) * xs + min(k + i % HALVES * 4 * N, depth - 1);
    };
    const auto fetch = [&](int k) {
      k += N * q;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (TINY) {
          if constexpr (TRANSPOSED) wp[i] = load_piece<T>(w + (int64_t)(n0 + i) * a.outer + k, n0 + i < width ? depth - k : 0);
          else wp[i] = load_piece<T>(w + (int64_t)(k + i) * a.outer + n0, k + i < depth ? width - n0 : 0);
        } else {
          const T* p = w_at(k, i);
          wp[i] = *reinterpret_cast<const typename Piece<T>::U*>(p + N <= w_end ? p : w_end - N);
        }
      }
#pragma unroll
      for (int r = 0; r < RB * HALVES; ++r) {
        if constexpr (TINY) {
          xp[r] = load_piece<T>(x + row[r] * xs + k, row[r] >= 0 ? depth - k : 0);
        } else {
          const T* p = x_at(k, r);
          xp[r] = *reinterpret_cast<const typename Piece<T>::U*>(p + N <= x_end ? p : x_end - N);
        }
      }
    };
    // near the contraction's end: what lies behind it
    const auto clear = [&](int k) {
      k += N * q;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned by = over(w_at(k, i), w_end);
        if (__any(by)) wp[i] = shifted<T>(wp[i], by);
        wp[i] = first_elements<T>(wp[i], TRANSPOSED ? depth - k - i % HALVES * 4 * N : k + i < depth ? N : 0);
      }
#pragma unroll
      for (int r = 0; r < RB * HALVES; ++r) {
        const unsigned by = over(x_at(k, r), x_end);
        if (__any(by)) xp[r] = shifted<T>(xp[r], by);
        xp[r] = first_elements<T>(xp[r], depth - k - r % HALVES * 4 * N);
      }
    };
    int k = wave * 4 * N * HALVES;
    if (k < depth) fetch(k);
    while (k < depth) {
      if (!TINY && k + 4 * N * HALVES + N > depth) clear(k);
      PieceV<T> wn[N], xn[RB * HALVES];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if constexpr (TRANSPOSED) {
          wn[j] = wp[j];
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) wn[j][i] = wp[i][j];
        }
      }
#pragma unroll
      for (int r = 0; r < RB * HALVES; ++r) xn[r] = xp[r];
      k += STEP;
      if (k < depth) fetch(k);
#pragma unroll
      for (int h = 0; h < HALVES; ++h)
#pragma unroll
        for (int j = 0; j < COLS; ++j)
#pragma unroll
          for (int r = 0; r < RB; ++r) acc[r][j] = multiply(wn[j * HALVES + h], xn[r * HALVES + h], acc[r][j]);
    }
  }
  const T *gate = (const T*)a.gate, *gate_end = gate + (int64_t)(a.rows - 1) * a.gs + width;
  T* y = (T*)a.y;
  // wave w ends up with the four columns' quarter w of every row block: columns col + COLS (4 q + w) .. + COLS - 1
  const int n = col + COLS * (4 * q + (wave & 3));
  float bias[COLS];
#pragma unroll
  for (int j = 0; j < COLS; ++j)
    bias[j] = !TRANSPOSED && a.bias && gt.group < a.groups ? a.bias[(int64_t)gt.group * width + min(n + j, width - 1)] : 0.f;
  PieceV<T> open[RB];
  if (TRANSPOSED && gate && wave < 4) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      if constexpr (TINY) open[r] = load_piece<T>(gate + row[r] * a.gs + n, row[r] >= 0 ? width - n : 0);
      else open[r] = load_within<T>(gate + (row[r] < 0 ? 0 : row[r]) * a.gs + min(n, width - 1), gate_end);
    }
  }
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    if (r) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < COLS; ++j) meet[wave][i][lane][j] = acc[r][j][i];
    __syncthreads();
    if (wave < 4 && row[r] >= 0 && n < width) {
      PieceV<T> out = {};
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        float v = bias[j];
#pragma unroll
        for (int s = 0; s < WAVES; ++s) v += meet[s][wave & 3][lane][j];
        if (!TRANSPOSED && a.relu) v = v < 0.f ? 0.f : v;   // (a NaN stays one)
        if (TRANSPOSED && gate) v = (float)open[r][j] > 0.f ? v : 0.f;
        out[j] = (T)v;
      }
      T* to = y + row[r] * a.ys + n;
      if constexpr (COLS == N) store_piece<T>(to, out, width - n);
      else store_first<T>(to, out, min(width - n, COLS));
    }
  }
}

// dW and db of a group: 16 N outer by 8 N inner columns to a workgroup, the waves share the group's rows; or (SHARED false, for groups of a few rows, which
// would keep one wave of four busy) a quarter as many inner columns to a wave, whose results leave from its registers. Both operands
// run across the contraction (the rows), so both are turned around in registers. db is one more product, with ones for x. The rows
// of the next step are looked up, and those of this one's are on their way, while the products of the one before are formed. Bound by the latency of those loads,
// about 2 us a step, and a group's rows are never cut over workgroups: long groups belong to the tiles.
template <typename T, bool SHARED, bool TINY>
__global__ __launch_bounds__(64 * kWaves) void few_rows_weights_kernel(MmArgs a) {
  constexpr int N = Piece<T>::N, H = SHARED ? N / 2 : N / 4, STEP = (SHARED ? kWaves : 1) * 4 * N;
  typedef T Half __attribute__((ext_vector_type(H)));
  typedef T HalfU __attribute__((ext_vector_type(H), aligned(sizeof(T))));
  __shared__ float meet[SHARED ? kWaves : 1][4][64][N];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, m = lane & 15, q = lane >> 4;
  const int group = (int)blockIdx.y;
  const int col = ((int)blockIdx.x % a.col_tiles) * 16 * N, in0 = ((int)blockIdx.x / a.col_tiles * (SHARED ? 1 : kWaves) + (SHARED ? 0 : wave)) * 16 * H;
  if (!SHARED && in0 >= a.inner) return;
  int begin, end;
  ds_group_range(a.offsets, a.groups, a.rows, group, &begin, &end);
  const T *x = (const T*)a.x, *dy = (const T*)a.dy;
  const T *x_end = x + (int64_t)(a.rows - 1) * a.xs + a.inner, *dy_end = dy + (int64_t)(a.rows - 1) * a.dys + a.outer;
  const int n0 = min(col + N * m, a.outer - 1), c0 = min(in0 + H * m, a.inner - 1);   // the lane's columns
  f32x4 acc[H][N] = {}, sum[N] = {};
  PieceV<T> ones;
#pragma unroll
  for (int i = 0; i < N; ++i) ones[i] = (T)1.f;
  const bool with_sum = in0 == 0;
  int row[N], late[N];   // of the pieces under way, and of the next ones
  PieceV<T> dp[N];
  Half xp[N];
  const auto look_up = [&](int at) {
#pragma unroll
    for (int i = 0; i < N; ++i) late[i] = at + N * q + i < end ? ds_ordered_row(a.order, a.rows, at + N * q + i) : -1;
  };
  const auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      row[i] = late[i];
      if constexpr (TINY) {
        dp[i] = load_piece<T>(dy + row[i] * a.dys + col + N * m, row[i] >= 0 ? a.outer - col - N * m : 0);
        const int have = row[i] >= 0 ? a.inner - in0 - H * m : 0;
#pragma unroll
        for (int j = 0; j < H; ++j) xp[i][j] = j < have ? x[row[i] * a.xs + in0 + H * m + j] : (T)0.f;
      } else {
        const int r = row[i] < 0 ? 0 : row[i];
        const T *pd = dy + r * a.dys + n0, *px = x + r * a.xs + c0;
        dp[i] = *reinterpret_cast<const typename Piece<T>::U*>(pd + N <= dy_end ? pd : dy_end - N);
        xp[i] = *reinterpret_cast<const HalfU*>(px + H <= x_end ? px : x_end - H);
      }
    }
  };
  int at = begin + (SHARED ? wave * 4 * N : 0);
  if (at < end) {
    look_up(at);
    fetch();
    if (at + STEP < end) look_up(at + STEP);
  }
  for (; at < end; at += STEP) {
    PieceV<T> dn[N], xn[H];
    if constexpr (!TINY) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        // (rows that there are not are cleared; pieces that would reach over the end have been read so that they end there)
        const int r = row[i] < 0 ? 0 : row[i];
        const int64_t by = dy + r * a.dys + n0 + N - dy_end, bx = x + r * a.xs + c0 + H - x_end;
        if (__any(by > 0)) dp[i] = shifted<T>(dp[i], by <= 0 ? 0 : by < N ? (unsigned)by : N);
        if (__any(bx > 0)) {
          Half moved = xp[i];
#pragma unroll
          for (int s = 1; s <= H; ++s)
            if (bx >= s) {
#pragma unroll
              for (int j = 0; j + 1 < H; ++j) moved[j] = moved[j + 1];
              moved[H - 1] = (T)0.f;
            }
          xp[i] = moved;
        }
        if (row[i] < 0) {
          dp[i] = PieceV<T>{};
          xp[i] = Half{};
        }
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int j = 0; j < N; ++j) dn[j][i] = dp[i][j];
#pragma unroll
      for (int j = 0; j < H; ++j) xn[j][i] = xp[i][j];
    }
    if (at + STEP < end) {
      fetch();
      if (at + 2 * STEP < end) look_up(at + 2 * STEP);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
#pragma unroll
      for (int h = 0; h < H; ++h) acc[h][j] = multiply(dn[j], xn[h], acc[h][j]);
      if (with_sum) sum[j] = multiply(dn[j], ones, sum[j]);
    }
  }
  T* dw = (T*)a.dw + (int64_t)group * a.inner * a.outer;
  if constexpr (!SHARED) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int in = in0 + H * m + h;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        PieceV<T> out;
#pragma unroll
        for (int j = 0; j < N; ++j) out[j] = (T)acc[h][j][i];
        const int n = col + N * (4 * q + i);
        if (in < a.inner && n < a.outer) store_piece<T>(dw + (int64_t)in * a.outer + n, out, a.outer - n);
      }
    }
    if (with_sum && m == 0) {   // (every column of the product with ones is the sum)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int n = col + N * (4 * q + i) + j;
          if (n < a.outer) a.db[(int64_t)group * a.outer + n] = sum[j][i];
        }
    }
    return;
  }
  const int n = col + N * (4 * q + wave);
#pragma unroll
  for (int h = 0; h <= H; ++h) {
    if (h == H && !with_sum) break;
    if (h) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) meet[wave][i][lane][j] = h < H ? acc[h < H ? h : 0][j][i] : sum[j][i];
    __syncthreads();
    float v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      v[j] = 0.f;
#pragma unroll
      for (int s = 0; s < kWaves; ++s) v[j] += meet[s][wave][lane][j];
    }
    if (h < H) {
      PieceV<T> out;
#pragma unroll
      for (int j = 0; j < N; ++j) out[j] = (T)v[j];
      const int in = in0 + H * m + h;
      if (in < a.inner && n < a.outer) {
        T* to = dw + (int64_t)in * a.outer + n;
        if (n + N <= a.outer) *reinterpret_cast<typename Piece<T>::U*>(to) = out;
        else store_first<T>(to, out, a.outer - n);
      }
    } else if (m == 0) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (n + j < a.outer) a.db[(int64_t)group * a.outer + n + j] = v[j];
    }
  }
}

MmArgs arguments(const ds_grouped& p) {
  MmArgs a = {};
  a.rows = p.rows;
  a.inner = p.inner;
  a.outer = p.outer;
  a.groups = p.groups;
  a.w = p.w;
  a.offsets = p.offsets;
  a.order = p.order;
  return a;
}

ds_mm_sizes sizes(const ds_grouped& p) { return {p.rows, p.inner, p.outer, p.groups}; }

// whether a matrix has less than 16 bytes from its first element to its last
template <typename T>
bool tiny_matrix(int64_t stride, int64_t rows, int64_t cols) {
  return (rows - 1) * stride + cols < Piece<T>::N;
}

template <typename T>
int element_of() {
  return sizeof(T) == 4 ? DS_ELEM_F32 : std::is_same<T, __bf16>::value ? DS_ELEM_BF16 : DS_ELEM_F16;
}

template <typename T, bool TRANSPOSED, bool HALF>
void launch_few(const ds_few_form& form, int64_t workgroups, const MmArgs& a, hipStream_t stream) {
  const dim3 block(64 * kWaves), twice(64 * 8);
  const ds_lines lines = ds_launch_lines(workgroups, 64 * (form.eight_waves ? 8 : kWaves));
  const dim3 grid(lines.x, lines.y);
  if (form.shift == 4 && form.eight_waves) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_kernel<T, 1, 8, TRANSPOSED, HALF, false>), dim3(grid), twice, 0, stream, a);
  else if (form.shift == 4) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_kernel<T, 1, kWaves, TRANSPOSED, HALF, false>), dim3(grid), block, 0, stream, a);
  else if (form.shift == 5 && form.eight_waves) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_kernel<T, 2, 8, TRANSPOSED, HALF, false>), dim3(grid), twice, 0, stream, a);
  else if (form.shift == 5) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_kernel<T, 2, kWaves, TRANSPOSED, HALF, false>), dim3(grid), block, 0, stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_kernel<T, 4, kWaves, TRANSPOSED, HALF, false>), dim3(grid), block, 0, stream, a);
}

template <typename T, bool TRANSPOSED>
int launch_rows(ds_ctx* ctx, const ds_grouped& p, MmArgs& a) {
  if (p.rows == 0) return DS_OK;
  hipStream_t stream = ctx->stream;
  // (rows of at least 16 bytes each would not be enough to ask for: an operand may have one row)
  const bool tiny = tiny_matrix<T>(TRANSPOSED ? a.dys : a.xs, p.rows, TRANSPOSED ? p.outer : p.inner) ||
                    tiny_matrix<T>((int64_t)p.inner * p.outer, p.groups, (int64_t)p.inner * p.outer) || (a.gate && tiny_matrix<T>(a.gs, p.rows, p.inner));
  const int depth = TRANSPOSED ? p.outer : p.inner, width = TRANSPOSED ? p.inner : p.outer;
  if (ds_rows_in_tiles(sizes(p), element_of<T>(), depth, width)) return ds_launch_row_tiles(ctx, element_of<T>(), TRANSPOSED, a);
  const ds_few_form form = ds_choose_few(sizes(p), element_of<T>(), TRANSPOSED, tiny);
  a.col_tiles = (width + form.cols - 1) / form.cols;
  const int64_t tiles = ds_most_tiles(a, form.shift) * a.col_tiles;
  if (tiles > 0x7fff0000) return ds_fail(ctx, DS_EINVAL, "%d rows by %d columns are more tiles than a launch has", p.rows, width);
  const ds_lines lines = ds_launch_lines(tiles, 64 * kWaves);
  if (tiny) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_kernel<T, 4, kWaves, TRANSPOSED, false, true>), dim3(lines.x, lines.y), dim3(64 * kWaves), 0, stream, a);
  else if (form.half) launch_few<T, TRANSPOSED, TRANSPOSED>(form, tiles, a, stream);
  else launch_few<T, TRANSPOSED, false>(form, tiles, a, stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

template <typename T>
int launch_weights(ds_ctx* ctx, const ds_grouped& p, MmArgs& a) {
  constexpr int N = Piece<T>::N;
  a.col_tiles = (p.outer + 16 * N - 1) / (16 * N);
  const bool shared = ds_weights_shared(sizes(p));
  const bool tiny = tiny_matrix<T>(a.xs, p.rows, p.inner) || tiny_matrix<T>(a.dys, p.rows, p.outer);
  const int width = shared || tiny ? 8 * N : 16 * N;   // inner columns of a workgroup
  const int64_t tiles = (int64_t)((p.inner + width - 1) / width) * a.col_tiles;
  if (tiles > ds_most_workgroups(64 * kWaves))
    return ds_fail(ctx, DS_EINVAL, "weights of %d by %d are more tiles than a launch has", p.inner, p.outer);
  const dim3 grid((unsigned)tiles, p.groups), block(64 * kWaves);
  if (tiny) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_weights_kernel<T, true, true>), grid, block, 0, ctx->stream, a);
  else if (shared) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_weights_kernel<T, true, false>), grid, block, 0, ctx->stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(few_rows_weights_kernel<T, false, false>), grid, block, 0, ctx->stream, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

template <typename T>
int backward(ds_ctx* ctx, const ds_grouped& p, MmArgs& a, void* workspace) {
  DS_TRY((launch_rows<T, true>(ctx, p, a)));
  if (ds_weights_in_tiles(sizes(p), element_of<T>())) return ds_launch_weight_tiles(ctx, element_of<T>(), a, workspace);
  return launch_weights<T>(ctx, p, a);
}

}  // namespace

int ds_launch_grouped_mm(ds_ctx* ctx, int dtype, const ds_grouped& p, ds_rows x, const float* bias, int relu, ds_rows y) {
  if (p.rows == 0) return DS_OK;
  MmArgs a = arguments(p);
  a.x = x.data;
  a.xs = x.stride;
  a.bias = bias;
  a.relu = relu;
  a.y = (void*)y.data;
  a.ys = y.stride;
  if (dtype == DS_ELEM_F32) return launch_rows<float, false>(ctx, p, a);
  if (dtype == DS_ELEM_BF16) return launch_rows<__bf16, false>(ctx, p, a);
  return launch_rows<_Float16, false>(ctx, p, a);
}

int64_t ds_grouped_mm_backward_bytes(int dtype, const ds_grouped& p) {
  return ds_weights_in_tiles(sizes(p), dtype) ? ds_weight_tiles_bytes(dtype, p.rows, p.inner, p.outer) : 0;
}

int ds_launch_grouped_mm_backward(ds_ctx* ctx, int dtype, const ds_grouped& p, ds_rows dy, ds_rows x, ds_rows gate, ds_rows dx,
                                  void* dw, float* db, void* workspace) {
  MmArgs a = arguments(p);
  a.dy = dy.data;
  a.dys = dy.stride;
  a.x = x.data;
  a.xs = x.stride;
  a.gate = gate.data;
  a.gs = gate.stride;
  a.y = (void*)dx.data;
  a.ys = dx.stride;
  a.dw = dw;
  a.db = db;
  if (dtype == DS_ELEM_F32) return backward<float>(ctx, p, a, workspace);
  if (dtype == DS_ELEM_BF16) return backward<__bf16>(ctx, p, a, workspace);
  return backward<_Float16>(ctx, p, a, workspace);
}
