// Dropout of feature rows, with an optional residual sum.
//
//   y(r, c) = residual(r, c) + (kept(r, c) ? x(r, c) * 65536 / (65536 - t) : 0),   t = round(65536 p)
//
// The mask is never stored: element (r, c) is kept where a 16-bit draw is not below t, and the draw is half c % 2 (the low
// one first) of word c % 8 / 2 of Philox4x32-10 under the counter (c / 8, r mod 2^32, r / 2^32, tag) and the key `seed`. The backward pass is the
// same function of the gradient. One generator call yields the eight draws of a 16-byte piece (two for fp32 rows), so
// the pass stays at the memory's speed: eight elements cost about 20 wide multiplications.
#include "feature_ops.h"
#include "philox.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;

struct DropArgs {
  int64_t rows;
  int cols, calls;      // generator calls to a row: pieces of eight columns
  int64_t rows_step;    // how far a thread's next piece is: rows_step rows and calls_step pieces
  int calls_step;
  const void *x, *residual;
  void* y;
  int64_t xs, rs, ys;
  uint32_t seed_lo, seed_hi, tag, threshold;
  float scale;
};

// 16 bytes of a row of 16 or more (TINY: of fewer elements): those from `col` on, or the row's last ones, which settle moves to their place
// (element by element a row's end took as long as the rest: 131,072 rows of 1,021 bf16 with a residual 268 us, so 182; of 1,024 157)
template <typename T, bool TINY>
__device__ __forceinline__ PieceV<T> load_inside(const T* row, int col, int cols) {
  if constexpr (TINY) return load_piece<T>(row + col, cols - col);
  else return *reinterpret_cast<const typename Piece<T>::U*>(row + min(col, cols - Piece<T>::N));
}
template <typename T, bool TINY>
__device__ __forceinline__ void settle(PieceV<T>& v, int col, int cols) {
  if (!TINY && cols - col < Piece<T>::N) v = shifted<T>(v, (unsigned)(col + Piece<T>::N - cols));
}

// Bound by memory: 131,072 rows of 1,024 bf16 with a residual 155 us, 5.19 TB/s (a large copy: 5.14). Workgroups stay, eight to a compute unit, and go
// through the pieces in steps of the whole grid; where the next piece lies is added, not divided.
template <typename T, bool RESIDUAL, bool TINY>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropArgs a) {
  constexpr int N = Piece<T>::N, PIECES = 8 / N;
  const uint32_t first = blockIdx.x * kThreads + threadIdx.x;
  int64_t row = first / (uint32_t)a.calls;
  int call = (int)(first % (uint32_t)a.calls);
  while (row < a.rows) {
    const int col = call * 8, have = a.cols - col;
    typename Piece<T>::V x[PIECES], r[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      x[p] = load_inside<T, TINY>((const T*)a.x + row * a.xs, col + p * N, a.cols);
      if constexpr (RESIDUAL) r[p] = load_inside<T, TINY>((const T*)a.residual + row * a.rs, col + p * N, a.cols);
    }
    uint32_t words[4];
    philox4x32_10((uint32_t)call, (uint32_t)row, (uint32_t)(row >> 32), a.tag, a.seed_lo, a.seed_hi, words);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      settle<T, TINY>(x[p], col + p * N, a.cols);
      if constexpr (RESIDUAL) settle<T, TINY>(r[p], col + p * N, a.cols);
      typename Piece<T>::V out;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = p * N + i;
        const uint32_t draw = e % 2 ? words[e / 2] >> 16 : words[e / 2] & 0xffffu;
        // (selected, not multiplied by zero: a dropped infinity or NaN leaves nothing)
        float v = draw >= a.threshold ? (float)x[p][i] * a.scale : 0.f;
        if constexpr (RESIDUAL) v = (float)r[p][i] + v;
        out[i] = (T)v;
      }
      store_piece<T>((T*)a.y + row * a.ys + col + p * N, out, have - p * N);
    }
    row += a.rows_step;
    call += a.calls_step;
    if (call >= a.calls) {
      call -= a.calls;
      ++row;
    }
  }
}

template <typename T>
void launch(const DropArgs& a, unsigned blocks, hipStream_t stream) {
  const dim3 grid(blocks), block(kThreads);
  if (a.cols < Piece<T>::N) {
    if (a.residual) hipLaunchKernelGGL(HIP_KERNEL_NAME(dropout_kernel<T, true, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(dropout_kernel<T, false, true>), grid, block, 0, stream, a);
  } else {
    if (a.residual) hipLaunchKernelGGL(HIP_KERNEL_NAME(dropout_kernel<T, true, false>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL(HIP_KERNEL_NAME(dropout_kernel<T, false, false>), grid, block, 0, stream, a);
  }
}

}  // namespace

int ds_launch_dropout(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows x, ds_rows residual, int threshold, uint64_t seed,
                      uint32_t tag, ds_rows y) {
  if (rows == 0) return DS_OK;
  DropArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.calls = (cols + 7) / 8;
  const int64_t pieces = rows * a.calls, want = (pieces + kThreads - 1) / kThreads, most = 8 * (int64_t)ctx->num_cus;
  const int64_t blocks = want < most ? want : most, step = blocks * kThreads;
  a.rows_step = step / a.calls;
  a.calls_step = (int)(step % a.calls);
  a.x = x.data;
  a.xs = x.stride;
  a.residual = residual.data;
  a.rs = residual.stride;
  a.y = (void*)y.data;
  a.ys = y.stride;
  a.seed_lo = (uint32_t)seed;
  a.seed_hi = (uint32_t)(seed >> 32);
  a.tag = tag;
  a.threshold = (uint32_t)threshold;
  a.scale = threshold < 65536 ? (float)(65536.0 / (65536 - threshold)) : 0.f;
  if (dtype == DS_ELEM_F32) launch<float>(a, (unsigned)blocks, ctx->stream);
  else if (dtype == DS_ELEM_BF16) launch<__bf16>(a, (unsigned)blocks, ctx->stream);
  else launch<_Float16>(a, (unsigned)blocks, ctx->stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}
