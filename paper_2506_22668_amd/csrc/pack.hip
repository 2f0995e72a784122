// Rows into 8 bits and back: e4m3 codes with a power of two for every 32 columns (packed.h).
//
// The power is the smallest that leaves the block's finite values at or below 448. A value is off by at most 2^-4 of itself where it is 2^-6 of that power or more, and by at
// most 2^-10 of the power from 2^-9 of it on. Two things are kept exactly: which values are 0, since a ReLU's gate is read from the codes (what is smaller than 2^-9 of the
// power becomes that, the smallest code, with its sign), and what is finite: no value comes back larger than its type holds, infinities and NaN come back as NaN.
#include "feature_ops.h"
#include "packed.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256, kCols = 8;   // columns of a thread: four threads to a block

struct PackArgs {
  int64_t rows;
  int cols, calls;              // pieces of eight columns to a row (pack: the last block's four filled up)
  int64_t rows_step;            // how far a thread's next piece is
  int calls_step;
  const void* x;                // pack: in; unpack: out
  uint8_t *codes, *scales;
  int64_t xs, cs, ss;
};

__device__ __forceinline__ uint32_t max_of_four(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
}

typedef uint32_t Eight __attribute__((ext_vector_type(2)));
typedef uint32_t EightU __attribute__((ext_vector_type(2), aligned(1)));

constexpr int kAhead = 2;   // pieces of a thread on their way at a time

// Most pieces take a product and half a conversion a value; those that hold a value which is not finite, which would round to 0, or near the type's largest
// go through the definition. Bound by memory, and for some of the inputs by vector instructions: 131,072 rows of 1,024 bf16
// 82 to 90 us, 4.5 to 4.9 TB/s (all through the definition: 104).
template <typename T, bool TINY>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackArgs a) {
  constexpr uint32_t kMostExponent = std::is_same<T, _Float16>::value ? 142 : 254;
  const int64_t first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int64_t row = first / a.calls;
  int call = (int)(first % a.calls);
  while (row < a.rows) {   // (the four threads of a block go on together)
    int64_t at[kAhead];
    int which[kAhead];
    typename Elements<T, kCols>::V v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      at[j] = row;
      which[j] = call;
      if (row < a.rows && call * kCols < a.cols) v[j] = load_elements<T, kCols, TINY>((const T*)a.x + row * a.xs, call * kCols, a.cols);
      row += a.rows_step;
      call += a.calls_step;
      if (call >= a.calls) {
        call -= a.calls;
        ++row;
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (at[j] >= a.rows) break;
      const int col = which[j] * kCols, have = a.cols - col;
      float x[kCols] = {};
      if (have >= kCols) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) x[i] = (float)v[j][i];
      } else if (have > 0) {
        settle_elements<T, kCols, TINY>(v[j], col, a.cols);
#pragma unroll
        for (int i = 0; i < kCols; ++i) x[i] = i < have ? (float)v[j][i] : 0.f;
      }
      uint32_t most = 0, least = 0xffffffffu;   // of the values' bits without a sign; of those that are not 0, less 1
#pragma unroll
      for (int i = 0; i < kCols; ++i) {
        const uint32_t bits = __float_as_uint(x[i]) & 0x7fffffffu;
        most = max(most, bits);
        least = min(least, bits - 1);
      }
      const bool fine = most < 0x7f800000u;
      if (!fine) {
        most = 0;
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          const uint32_t bits = __float_as_uint(x[i]) & 0x7fffffffu;
          most = max(most, bits < 0x7f800000u ? bits : 0);
        }
      }
      most = max_of_four(most);
      const uint32_t exponent = most >> 23;
      const bool wide = (most & 0x7fffffu) > 0x600000u;   // above 448 of the power below
      const uint32_t scale = most == 0 ? 127 : max((int)exponent - 8 + (int)wide, 1);
      const bool high = wide && exponent == kMostExponent;
      const float inv = __uint_as_float((254 - scale) << 23);
      const uint32_t smallest = __float_as_uint(power_of_scale(scale) * 0x1p-9f);   // the bits of what the smallest code stands for
      uint32_t word[2];
      if (fine && !high && least >= smallest - 1) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          word[w] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w] * inv, x[4 * w + 1] * inv, 0, false);
          word[w] = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * w + 2] * inv, x[4 * w + 3] * inv, word[w], true);
        }
      } else {
        const float top = high ? 240.f : 448.f;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          float q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float from = x[4 * w + i], s = from * inv;
            q[i] = fabsf(s) < 0x1p-9f && from != 0.f ? copysignf(0x1p-9f, from) : fminf(fmaxf(s, -top), top);
            if (!(fabsf(from) < INFINITY)) q[i] = NAN;
          }
          word[w] = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
          word[w] = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], word[w], true);
        }
      }
      uint8_t* to = a.codes + at[j] * a.cs + col;
      if (have >= kCols) {
        *reinterpret_cast<EightU*>(to) = Eight{word[0], word[1]};
      } else {
#pragma unroll
        for (int i = 0; i < kCols - 1; ++i)
          if (i < have) to[i] = (uint8_t)(word[i / 4] >> (8 * (i % 4)));
      }
      if (which[j] % 4 == 0) a.scales[at[j] * a.ss + which[j] / 4] = (uint8_t)scale;
    }
  }
}

// Bound by memory: 131,072 rows of 1,024 bf16 67 us, 6.1 TB/s (the codes were packed right before, and come from the cache in part).
template <typename T>
__global__ __launch_bounds__(kThreads) void unpack_kernel(PackArgs a) {
  constexpr int N = Piece<T>::N;
  const int64_t first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int64_t row = first / a.calls;
  int call = (int)(first % a.calls);
  while (row < a.rows) {
    const int col = call * kCols, have = a.cols - col;
    const uint8_t* from = a.codes + row * a.cs + col;
    uint32_t word[2] = {0, 0};
    if (have >= kCols) {
      const Eight v = *reinterpret_cast<const EightU*>(from);
      word[0] = v[0];
      word[1] = v[1];
    } else {
#pragma unroll
      for (int i = 0; i < kCols - 1; ++i)
        if (i < have) word[i / 4] |= (uint32_t)from[i] << (8 * (i % 4));
    }
    const float power = power_of_scale(a.scales[row * a.ss + col / kPackBlock]);
    float x[kCols];
#pragma unroll
    for (int i = 0; i < kCols; i += 2) {
      const auto two = i % 4 ? __builtin_amdgcn_cvt_pk_f32_fp8(word[i / 4], true) : __builtin_amdgcn_cvt_pk_f32_fp8(word[i / 4], false);
      x[i] = two[0] * power;
      x[i + 1] = two[1] * power;
    }
#pragma unroll
    for (int p = 0; p < kCols / N; ++p) {
      PieceV<T> out;
#pragma unroll
      for (int i = 0; i < N; ++i) out[i] = (T)x[p * N + i];
      store_piece<T>((T*)a.x + row * a.xs + col + p * N, out, have - p * N);
    }
    row += a.rows_step;
    call += a.calls_step;
    if (call >= a.calls) {
      call -= a.calls;
      ++row;
    }
  }
}

unsigned spread(ds_ctx* ctx, PackArgs& a, int calls) {
  a.calls = calls;
  const int64_t pieces = a.rows * a.calls, want = (pieces + kThreads - 1) / kThreads, most = 8 * (int64_t)ctx->num_cus;
  const int64_t blocks = want < most ? want : most, step = blocks * kThreads;
  a.rows_step = step / a.calls;
  a.calls_step = (int)(step % a.calls);
  return (unsigned)blocks;
}

template <typename T>
void launch_pack(const PackArgs& a, unsigned blocks, hipStream_t stream) {
  if (a.cols < kCols) hipLaunchKernelGGL(HIP_KERNEL_NAME(pack_kernel<T, true>), dim3(blocks), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(pack_kernel<T, false>), dim3(blocks), dim3(kThreads), 0, stream, a);
}

}  // namespace

int ds_launch_pack(ds_ctx* ctx, int dtype, int64_t rows, int cols, ds_rows x, const ds_packed& to) {
  if (rows == 0) return DS_OK;
  PackArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.x = x.data;
  a.xs = x.stride;
  a.codes = (uint8_t*)to.codes;
  a.cs = to.codes_stride;
  a.scales = (uint8_t*)to.scales;
  a.ss = to.scales_stride;
  const unsigned blocks = spread(ctx, a, (cols + kPackBlock - 1) / kPackBlock * (kPackBlock / kCols));
  if (dtype == DS_ELEM_F32) launch_pack<float>(a, blocks, ctx->stream);
  else if (dtype == DS_ELEM_BF16) launch_pack<__bf16>(a, blocks, ctx->stream);
  else launch_pack<_Float16>(a, blocks, ctx->stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

int ds_launch_unpack(ds_ctx* ctx, int dtype, int64_t rows, int cols, const ds_packed& from, ds_rows y) {
  if (rows == 0) return DS_OK;
  PackArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.x = y.data;
  a.xs = y.stride;
  a.codes = (uint8_t*)from.codes;
  a.cs = from.codes_stride;
  a.scales = (uint8_t*)from.scales;
  a.ss = from.scales_stride;
  const unsigned blocks = spread(ctx, a, (cols + kCols - 1) / kCols);
  if (dtype == DS_ELEM_F32) hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<float>), dim3(blocks), dim3(kThreads), 0, ctx->stream, a);
  else if (dtype == DS_ELEM_BF16) hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<__bf16>), dim3(blocks), dim3(kThreads), 0, ctx->stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(unpack_kernel<_Float16>), dim3(blocks), dim3(kThreads), 0, ctx->stream, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}
