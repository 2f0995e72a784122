// Layer norm of feature rows, forward and backward.
//
//   forward:   mu = mean_c x, rstd = 1 / sqrt(mean_c (x - mu)^2 + eps), y = (x - mu) rstd w + b
//   backward:  xhat = (x - mu) rstd, g = dy w,  dx = rstd (g - mean_c g - xhat mean_c (g xhat)),
//              dw = sum over rows of dy xhat, db = sum over rows of dy
//
// A row of up to 4,096 columns stays in the registers of TPR threads, 16 columns to a thread (TPR a power of two: part of a
// wave, a wave, or up to four), so it is read once and the variance is the mean of squares about the mean that is already known. All sums are
// fp32, whatever the rows' type; a result is rounded once.
#include "feature_ops.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;   // columns of a thread

struct NormArgs {
  int64_t rows;
  int cols;
  const void *x, *dy;
  int64_t xs, dys, ys;
  const float *weight, *bias, *mean_in, *rstd_in;
  float eps;
  void* y;
  float *mean, *rstd;   // out, or null
  float* partial;       // [block][2][cols]
  float *dweight, *dbias;   // where one workgroup takes all rows
};

// The columns of a thread: pieces of 16 bytes, a row's threads side by side
template <typename T, int TPR>
struct Columns {
  static constexpr int N = Piece<T>::N, PIECES = kPer / N;
  int at[PIECES], have[PIECES];
  int last;               // where the row's last 16 bytes begin; below zero: it has less
  __device__ __forceinline__ Columns(int t, int cols) : last(cols - N) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      at[p] = (p * TPR + t) * N;
      have[p] = cols - at[p];   // (not above zero: none)
    }
  }
};

template <typename T, int TPR>
struct Row {
  static constexpr int N = Piece<T>::N, PIECES = kPer / N;
  typename Piece<T>::V v[PIECES];
  // Every thread reads 16 bytes inside of the row, without a branch; settle, where they are used, moves those of the row's end to their place. (Element by
  // element, the row's end was waited for in front of the next row: 131,072 rows of 1,021 bf16 166 us, so 122; of 1,024 112.)
  __device__ __forceinline__ void load(const T* row, const Columns<T, TPR>& c) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      if (TPR == 2 && c.last < 0) v[p] = load_piece<T>(row + c.at[p], c.have[p]);
      else v[p] = *reinterpret_cast<const typename Piece<T>::U*>(row + min(c.at[p], c.last));
    }
  }
  __device__ __forceinline__ void settle(const Columns<T, TPR>& c) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      if (TPR == 2 && c.last < 0) continue;
      if (c.last % N && c.have[p] > 0 && c.have[p] < N) v[p] = shifted<T>(v[p], (unsigned)(c.at[p] - c.last));
      if (c.have[p] <= 0) v[p] = PieceV<T>{};
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) v[p] = typename Piece<T>::V{};
  }
};

// Sum over a row's threads, in all of them. Past a wave through LDS; `turn` alternates between two sets of slots, so that
// one barrier a sum is enough.
template <int TPR>
__device__ __forceinline__ void sum_row(float& a, float& b, float (*slots)[4][2], int& turn) {
  a = sum_lanes<(TPR < 64 ? TPR : 64)>(a);
  b = sum_lanes<(TPR < 64 ? TPR : 64)>(b);
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6, first = wave / (TPR / 64) * (TPR / 64);
    if ((threadIdx.x & 63) == 0) {
      slots[turn][wave][0] = a;
      slots[turn][wave][1] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < TPR / 64; ++i) {
      a += slots[turn][first + i][0];
      b += slots[turn][first + i][1];
    }
    turn ^= 1;
  }
}

template <typename T, int TPR>
__device__ __forceinline__ void load_params(const float* from, float absent, const Columns<T, TPR>& c, float (&to)[kPer]) {
  constexpr int N = Piece<T>::N;
#pragma unroll
  for (int i = 0; i < kPer; ++i) to[i] = from && i % N < c.have[i / N] ? from[c.at[i / N] + i % N] : absent;
}

// Bound by memory, a row read and written: 131,072 rows of 1,024 bf16 106 us, 5.06 TB/s (a large copy: 5.14); 33 rows of 256 fp32 7.4 us, of which the kernel takes 4.
// (The row after is on its way while this one's sums are formed.)
template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(NormArgs a) {
  constexpr int N = Piece<T>::N, PIECES = kPer / N, ROWS = kThreads / TPR;
  __shared__ float slots[2][4][2];
  int turn = 0;
  const int t = threadIdx.x % TPR;
  const Columns<T, TPR> c(t, a.cols);
  float w[kPer], b[kPer];
  load_params<T, TPR>(a.weight, 1.f, c, w);
  load_params<T, TPR>(a.bias, 0.f, c, b);
  const float inv = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  Row<T, TPR> next;
  if (row < a.rows) next.load((const T*)a.x + row * a.xs, c);
  else next.clear();
  // (all threads of a workgroup go round equally often: the sums of a wide row meet at barriers)
  for (int64_t base = (int64_t)blockIdx.x * ROWS; base < a.rows; base += step, row += step) {
    Row<T, TPR> x = next;
    x.settle(c);
    if (row + step < a.rows) next.load((const T*)a.x + (row + step) * a.xs, c);
    float s = 0.f, none = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s += (float)x.v[i / N][i % N];
    sum_row<TPR>(s, none, slots, turn);
    const float mean = s * inv;
    float d[kPer], q = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      d[i] = (float)x.v[i / N][i % N] - mean;
      if (i % N < c.have[i / N]) q = fmaf(d[i], d[i], q);
    }
    sum_row<TPR>(q, none, slots, turn);
    const float rstd = rsqrtf(fmaf(q, inv, a.eps));
    if (row < a.rows) {
      T* y = (T*)a.y + row * a.ys;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        typename Piece<T>::V out;
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = (T)fmaf(d[p * N + i] * rstd, w[p * N + i], b[p * N + i]);
        store_piece<T>(y + c.at[p], out, c.have[p]);
      }
      if (t == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

// dw and db: a thread adds up its columns over its rows in registers, the workgroup's rows meet in LDS, and every workgroup
// leaves one pair of partial rows: no atomics, so the same inputs give the same bits. Bound by memory (x and dy read, dx written): 100,003 rows of 1,000
// bf16 126 us, 4.8 TB/s, 30,011 rows of 515 fp32 49 us, 3.8 TB/s, of which the second launch and the gap before
// it take 12. 16-bit rows are kept to 128 registers, for four waves to a SIMD, though 3 to 13 of their values
// then go through scratch memory (133, three waves: 134 us; 400,000 rows of 130: 90 -> 71).
template <typename T, int TPR>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) void layer_norm_backward_kernel(NormArgs a) {
  constexpr int N = Piece<T>::N, PIECES = kPer / N, ROWS = kThreads / TPR;
  __shared__ float slots[2][4][2];
  __shared__ float meet[ROWS > 1 ? kThreads * kPer : 1];
  int turn = 0;
  const int t = threadIdx.x % TPR;
  const Columns<T, TPR> c(t, a.cols);
  float w[kPer], dw[kPer] = {}, db[kPer] = {};
  load_params<T, TPR>(a.weight, 1.f, c, w);
  const float inv = 1.f / (float)a.cols;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  Row<T, TPR> next_x, next_dy;
  float next_mean = 0.f, next_rstd = 0.f;
  const auto fetch = [&](int64_t r) {
    next_x.load((const T*)a.x + r * a.xs, c);
    next_dy.load((const T*)a.dy + r * a.dys, c);
    next_mean = a.mean_in[r];
    next_rstd = a.rstd_in[r];
  };
  next_x.clear();
  next_dy.clear();
  if (row < a.rows) fetch(row);
  for (int64_t base = (int64_t)blockIdx.x * ROWS; base < a.rows; base += step, row += step) {
    Row<T, TPR> x = next_x, dy = next_dy;
    x.settle(c);
    dy.settle(c);
    const float mean = next_mean, rstd = next_rstd;
    const bool live = row < a.rows;
    if (row + step < a.rows) fetch(row + step);
    float hat[kPer], s = 0.f, p = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float g = (float)dy.v[i / N][i % N];
      hat[i] = ((float)x.v[i / N][i % N] - mean) * rstd;
      if (live && i % N < c.have[i / N]) {
        dw[i] = fmaf(g, hat[i], dw[i]);
        db[i] += g;
        s = fmaf(g, w[i], s);
        p = fmaf(g * w[i], hat[i], p);
      }
    }
    sum_row<TPR>(s, p, slots, turn);
    s *= inv;
    p *= inv;
    if (live) {
      T* dx = (T*)a.y + row * a.ys;
#pragma unroll
      for (int q = 0; q < PIECES; ++q) {
        typename Piece<T>::V out;
#pragma unroll
        for (int i = 0; i < N; ++i)
          out[i] = (T)(rstd * (fmaf((float)dy.v[q][i], w[q * N + i], -s) - hat[q * N + i] * p));
        store_piece<T>(dx + c.at[q], out, c.have[q]);
      }
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* to = gridDim.x == 1 ? which ? a.dbias : a.dweight : a.partial + ((int64_t)blockIdx.x * 2 + which) * a.cols;
    const float(&v)[kPer] = which ? db : dw;
    if constexpr (ROWS == 1) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (i % N < c.have[i / N]) to[c.at[i / N] + i % N] = v[i];
    } else {
      const int slot = threadIdx.x / TPR;
      if (which) __syncthreads();
#pragma unroll
      for (int i = 0; i < kPer; ++i) meet[slot * (TPR * kPer) + c.at[i / N] + i % N] = v[i];
      __syncthreads();
      for (int col = threadIdx.x; col < a.cols; col += kThreads) {
        float sum = 0.f;
#pragma unroll 8
        for (int r = 0; r < ROWS; ++r) sum += meet[r * (TPR * kPer) + col];
        to[col] = sum;
      }
    }
  }
}

// The partial rows of all workgroups, in a fixed order: 32 columns to a workgroup, 32 threads to a column
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const float* partial, int parts, int cols, float* dweight,
                                                               float* dbias) {
  __shared__ float meet[32][33];
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, width = 2 * cols;
  const int col = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < width) {
#pragma unroll 8
    for (int i = part; i < parts; i += 32) s += partial[(int64_t)i * width + col];
  }
  meet[part][lane] = s;
  __syncthreads();
  if (part == 0 && col < width) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += meet[i][lane];
    if (col < cols) dweight[col] = s;
    else dbias[col - cols] = s;
  }
}

// threads to a row: the fewest that hold it
int threads_of_row(int cols) {
  int t = 2;
  while (t * kPer < cols) t *= 2;
  return t;
}

template <typename T, int TPR>
void launch(bool backward, const NormArgs& a, unsigned blocks, hipStream_t stream) {
  if (backward) hipLaunchKernelGGL(HIP_KERNEL_NAME(layer_norm_backward_kernel<T, TPR>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(layer_norm_kernel<T, TPR>), dim3(blocks), dim3(kThreads), 0, stream, a);
}

template <typename T>
void launch_for(bool backward, const NormArgs& a, unsigned blocks, hipStream_t stream) {
  switch (threads_of_row(a.cols)) {
    case 2: return launch<T, 2>(backward, a, blocks, stream);
    case 4: return launch<T, 4>(backward, a, blocks, stream);
    case 8: return launch<T, 8>(backward, a, blocks, stream);
    case 16: return launch<T, 16>(backward, a, blocks, stream);
    case 32: return launch<T, 32>(backward, a, blocks, stream);
    case 64: return launch<T, 64>(backward, a, blocks, stream);
    case 128: return launch<T, 128>(backward, a, blocks, stream);
    default: return launch<T, 256>(backward, a, blocks, stream);
  }
}

int run(ds_ctx* ctx, bool backward, int dtype, const NormArgs& a, int64_t blocks) {
  if (dtype == DS_ELEM_F32) launch_for<float>(backward, a, (unsigned)blocks, ctx->stream);
  else if (dtype == DS_ELEM_BF16) launch_for<__bf16>(backward, a, (unsigned)blocks, ctx->stream);
  else launch_for<_Float16>(backward, a, (unsigned)blocks, ctx->stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

int64_t blocks_for(int64_t rows, int cols, int64_t most) {
  const int64_t per = kThreads / threads_of_row(cols), blocks = (rows + per - 1) / per;
  return blocks < most ? blocks : most;
}

}  // namespace

int ds_launch_layer_norm(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows x, const float* weight, const float* bias,
                         float eps, ds_rows y, float* mean, float* rstd) {
  if (rows == 0) return DS_OK;
  NormArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.x = x.data;
  a.xs = x.stride;
  a.y = (void*)y.data;
  a.ys = y.stride;
  a.weight = weight;
  a.bias = bias;
  a.eps = eps;
  a.mean = mean;
  a.rstd = rstd;
  return run(ctx, false, dtype, a, blocks_for(rows, cols, 8 * (int64_t)ctx->num_cus));
}

// Up to four rows to a thread one workgroup takes them all, and there is nothing to add up (64 rows of 256 bf16 17.5 -> 14.6 us, 4 of 4,096 17.4 -> 15.2;
// eight rows to a thread: 128 of 256 17.5 -> 14.5, but 8 of 4,096 17.6 -> 23).
constexpr int kAlone = 4;
int64_t ds_layer_norm_partials(int64_t rows, int cols) {
  return rows <= kAlone * (int64_t)(kThreads / threads_of_row(cols)) ? 1 : blocks_for(rows, cols, 1024);
}

int ds_launch_layer_norm_backward(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows dy, ds_rows x, const float* mean,
                                  const float* rstd, const float* weight, ds_rows dx, float* dweight, float* dbias,
                                  float* partial) {
  const int64_t parts = ds_layer_norm_partials(rows, cols);
  if (rows > 0) {
    NormArgs a = {};
    a.rows = rows;
    a.cols = cols;
    a.x = x.data;
    a.xs = x.stride;
    a.dy = dy.data;
    a.dys = dy.stride;
    a.y = (void*)dx.data;
    a.ys = dx.stride;
    a.weight = weight;
    a.mean_in = mean;
    a.rstd_in = rstd;
    a.partial = partial;
    a.dweight = dweight;
    a.dbias = dbias;
    DS_TRY(run(ctx, true, dtype, a, parts));
    if (parts == 1) return DS_OK;
  }
  hipLaunchKernelGGL(layer_norm_join_kernel, dim3((2 * cols + 31) / 32), dim3(1024), 0, ctx->stream, partial, rows > 0 ? (int)parts : 0, cols,
                     dweight, dbias);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}
