// The experts of every row from a router's scores, how evenly they are used, and the scores' gradient.
//
//   forward:   p = softmax(x) over a row's experts; ids: those of the k highest scores, ties to the lowest, -inf never; w_j = p at id_j, or its share of
//              the k; counts_e = how often e was chosen, N = rows with an expert; loss = E sum_e (counts_e / sum of counts) (sum_r p_re / N)
//   backward:  dx = p (g - sum_e p g), g_e = dloss E counts_e / (N sum of counts) + [e = id_j] dp_j,
//              dp_j = dw_j, or (dw_j - sum_i dw_i w_i) / sum of the chosen p
//
// A row of up to 1,024 scores stays in the registers of TPR threads, 16 to a thread. A row that is -inf throughout has no expert: ids -1, weights 0, and it takes no
// part in N. One with NaN or +inf has none either, but its weights, and so the loss, are NaN. All sums are fp32, over rows first in a thread, then in
// a workgroup, and the workgroups' in 64 bits in a fixed order: the same inputs give the same bits.
#include <math.h>

#include "feature_ops.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;   // scores of a thread

struct RouteArgs {
  int64_t rows;
  int experts, k;
  bool renorm;
  const void* x;
  int64_t xs;
  int32_t* ids;
  float *weights, *loss, *lse;
  int64_t* counts;
  // what workgroups leave, where there are several: sums of p [block][experts], counts [block][experts], rows [block]
  float* sums;
  int32_t *chosen, *with;
};

template <int CTRL>
__device__ __forceinline__ int across(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
// The highest (lowest) of LANES neighbouring lanes, in each of them
template <int LANES>
__device__ __forceinline__ float max_lanes(float v) {
  if constexpr (LANES >= 2) v = fmaxf(v, __int_as_float(across<0xB1>(__float_as_int(v))));
  if constexpr (LANES >= 4) v = fmaxf(v, __int_as_float(across<0x4E>(__float_as_int(v))));
  if constexpr (LANES >= 8) v = fmaxf(v, __int_as_float(across<0x141>(__float_as_int(v))));
  if constexpr (LANES >= 16) v = fmaxf(v, __int_as_float(across<0x140>(__float_as_int(v))));
  if constexpr (LANES >= 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
  if constexpr (LANES >= 64) v = fmaxf(v, __shfl_xor(v, 32, 64));
  return v;
}
template <int LANES>
__device__ __forceinline__ int min_lanes(int v) {
  if constexpr (LANES >= 2) v = min(v, across<0xB1>(v));
  if constexpr (LANES >= 4) v = min(v, across<0x4E>(v));
  if constexpr (LANES >= 8) v = min(v, across<0x141>(v));
  if constexpr (LANES >= 16) v = min(v, across<0x140>(v));
  if constexpr (LANES >= 32) v = min(v, __shfl_xor(v, 16, 64));
  if constexpr (LANES >= 64) v = min(v, __shfl_xor(v, 32, 64));
  return v;
}

// A thread's scores: pieces of 16 bytes, a row's threads side by side; `absent` where the row has ended
template <typename T, int TPR>
struct Scores {
  static constexpr int N = Piece<T>::N, PIECES = kPer / N;
  PieceV<T> v[PIECES];
  __device__ __forceinline__ void load(const T* row, int t, int experts) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (p * TPR + t) * N;
      if (experts < N) v[p] = load_piece<T>(row + at, experts - at);
      else v[p] = *reinterpret_cast<const typename Piece<T>::U*>(row + min(at, experts - N));
    }
  }
  __device__ __forceinline__ void read(int t, int experts, float absent, float (&to)[kPer]) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (p * TPR + t) * N, have = experts - at;
      if (experts >= N && have > 0 && have < N) v[p] = shifted<T>(v[p], (unsigned)(N - have));
#pragma unroll
      for (int i = 0; i < N; ++i) to[p * N + i] = i < have ? (float)v[p][i] : absent;
    }
  }
};
// the expert of a thread's score i
template <typename T, int TPR>
__device__ __forceinline__ int expert_of(int t, int i) {
  constexpr int N = Piece<T>::N;
  return (i / N * TPR + t) * N + i % N;
}

template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
  constexpr int ROWS = kThreads / TPR;
  __shared__ float meet[kThreads * kPer];
  __shared__ int with_of[kThreads];
  const int t = threadIdx.x % TPR;
  const float none = -INFINITY;
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  float sum[kPer] = {};
  int took[kPer] = {}, with = 0;
  Scores<T, TPR> next = {};
  if (row < a.rows) next.load((const T*)a.x + row * a.xs, t, a.experts);
  for (; row < a.rows; row += step) {
    Scores<T, TPR> now = next;
    if (row + step < a.rows) next.load((const T*)a.x + (row + step) * a.xs, t, a.experts);
    float x[kPer];
    now.read(t, a.experts, none, x);
    float most = none;
#pragma unroll
    for (int i = 0; i < kPer; ++i) most = fmaxf(most, x[i]);
    most = max_lanes<TPR>(most);
    const float top = most == none ? 0.f : most;
    float q[kPer], total = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      q[i] = expf(x[i] - top);
      total += q[i];
    }
    total = sum_lanes<TPR>(total);
    const bool fine = total > 0.f && total < INFINITY;   // (a NaN is neither; a row without an open expert sums up to 0)
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < kPer; ++i) sum[i] = fmaf(q[i], inv, sum[i]);
    with += fine;
    float weight[8], shares = 0.f;
    int id[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= a.k) break;
      float best = none;
      int at = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (x[i] > best) {
          best = x[i];
          at = expert_of<T, TPR>(t, i);
        }
      const float high = max_lanes<TPR>(best);
      const int first = min_lanes<TPR>(best == high ? at : 0x7fffffff);
      const bool is = fine && high > none;
      id[j] = is ? first : -1;
      weight[j] = is ? expf(high - top) * inv : fine || total == 0.f ? 0.f : NAN;
      shares += weight[j];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const bool mine = is && first == expert_of<T, TPR>(t, i);
        x[i] = mine ? none : x[i];
        took[i] += mine;
      }
    }
    if (t == 0) {
      const float by = a.renorm && shares > 0.f ? 1.f / shares : 1.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= a.k) break;
        a.ids[j * a.rows + row] = id[j];
        a.weights[j * a.rows + row] = weight[j] * by;
      }
      if (a.lse) a.lse[row] = total == 0.f ? none : top + logf(total);
    }
  }
  // the workgroup's rows
  with_of[threadIdx.x] = t == 0 ? with : 0;
  const int slot = threadIdx.x / TPR;
  float* sums = a.sums + (int64_t)blockIdx.x * a.experts;
  int32_t* chosen = a.chosen + (int64_t)blockIdx.x * a.experts;
#pragma unroll
  for (int i = 0; i < kPer; ++i) meet[slot * (TPR * kPer) + expert_of<T, TPR>(t, i)] = sum[i];
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    float s = 0.f;
    for (int r = 0; r < ROWS; ++r) s += meet[r * (TPR * kPer) + e];
    sums[e] = s;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kPer; ++i) meet[slot * (TPR * kPer) + expert_of<T, TPR>(t, i)] = __int_as_float(took[i]);
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    int s = 0;
    for (int r = 0; r < ROWS; ++r) s += __float_as_int(meet[r * (TPR * kPer) + e]);
    chosen[e] = s;
  }
  for (int o = kThreads / 2; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) with_of[threadIdx.x] += with_of[threadIdx.x + o];
    __syncthreads();
  }
  if (threadIdx.x == 0) a.with[blockIdx.x] = with_of[0];
}

// What the workgroups left, in order
__global__ __launch_bounds__(1024) void route_join_kernel(RouteArgs a, int blocks) {
  __shared__ double part[1024];
  __shared__ int64_t number[1024];
  double loss = 0.0;
  int64_t chosen = 0, with = 0;
  for (int e = threadIdx.x; e < a.experts; e += 1024) {
    double s = 0.0;
    int64_t n = 0;
    for (int b = 0; b < blocks; ++b) {
      s += a.sums[(int64_t)b * a.experts + e];
      n += a.chosen[(int64_t)b * a.experts + e];
    }
    a.counts[e] = n;
    loss += s * (double)n;
    chosen += n;
  }
  for (int b = threadIdx.x; b < blocks; b += 1024) with += a.with[b];
  const auto all = [&](auto* slots, auto v) {
    slots[threadIdx.x] = v;
    __syncthreads();
    for (int o = 512; o > 0; o >>= 1) {
      if ((int)threadIdx.x < o) slots[threadIdx.x] += slots[threadIdx.x + o];
      __syncthreads();
    }
    const auto sum = slots[0];
    __syncthreads();
    return sum;
  };
  loss = all(part, loss);
  chosen = all(number, chosen);
  with = all(number, with);
  if (threadIdx.x == 0) {
    a.counts[a.experts] = with;
    // (a sum that is NaN stays one, where nothing was chosen too)
    *a.loss = (float)(loss * a.experts / ((double)(chosen > 0 ? chosen : 1) * (double)(with > 0 ? with : 1)));
  }
}

struct RouteGradArgs {
  int64_t rows;
  int experts, k;
  bool renorm;
  const void* x;
  int64_t xs, ys;
  const float *lse, *dweights, *dloss;
  const int32_t* ids;
  const int64_t* counts;
  void* dx;
};

template <typename T, int TPR>
__global__ __launch_bounds__(kThreads) void route_grad_kernel(RouteGradArgs a) {
  constexpr int ROWS = kThreads / TPR, N = Piece<T>::N, PIECES = kPer / N;
  __shared__ int64_t part[kThreads];
  const int t = threadIdx.x % TPR;
  const float none = -INFINITY;
  // the loss' part of g: the same for all rows
  float share[kPer] = {};
  if (a.dloss) {
    int64_t n = 0;
    for (int e = threadIdx.x; e < a.experts; e += kThreads) n += a.counts[e];
    part[threadIdx.x] = n;
    __syncthreads();
    for (int o = kThreads / 2; o > 0; o >>= 1) {
      if ((int)threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
      __syncthreads();
    }
    const int64_t chosen = part[0], with = a.counts[a.experts];
    const double by = (double)*a.dloss * a.experts / ((double)(chosen > 0 ? chosen : 1) * (double)(with > 0 ? with : 1));
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = expert_of<T, TPR>(t, i);
      share[i] = e < a.experts ? (float)(by * (double)a.counts[e]) : 0.f;
    }
  }
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
  Scores<T, TPR> next = {};
  if (row < a.rows) next.load((const T*)a.x + row * a.xs, t, a.experts);
  for (; row < a.rows; row += step) {
    Scores<T, TPR> now = next;
    if (row + step < a.rows) next.load((const T*)a.x + (row + step) * a.xs, t, a.experts);
    float p[kPer], g[kPer];
    now.read(t, a.experts, none, p);
    const float lse = a.lse[row];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      p[i] = lse == none ? 0.f : expf(p[i] - lse);
      g[i] = share[i];
    }
    if (a.dweights) {
      int id[8];
      float dw[8], of[8], dot = 0.f, total = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= a.k) break;
        id[j] = a.ids[j * a.rows + row];
        dw[j] = a.dweights[j * a.rows + row];
        if ((uint32_t)id[j] >= (uint32_t)a.experts) id[j] = -1;
        if (a.renorm) {
          float mine = 0.f;
#pragma unroll
          for (int i = 0; i < kPer; ++i) mine = id[j] == expert_of<T, TPR>(t, i) ? p[i] : mine;
          of[j] = sum_lanes<TPR>(mine);
          total += of[j];
          if (id[j] >= 0) dot = fmaf(dw[j], of[j], dot);
        }
      }
      const float inv = a.renorm ? total > 0.f ? 1.f / total : 0.f : 1.f;
      dot *= inv;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= a.k) break;
        const float dp = (dw[j] - dot) * inv;
#pragma unroll
        for (int i = 0; i < kPer; ++i) g[i] += id[j] == expert_of<T, TPR>(t, i) ? dp : 0.f;
      }
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s = fmaf(p[i], g[i], s);
    s = sum_lanes<TPR>(s);
    T* dx = (T*)a.dx + row * a.ys;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
      const int at = (q * TPR + t) * N;
      PieceV<T> out;
#pragma unroll
      for (int i = 0; i < N; ++i) out[i] = (T)(p[q * N + i] * (g[q * N + i] - s));
      store_piece<T>(dx + at, out, a.experts - at);
    }
  }
}

int threads_of_row(int experts) {
  int t = 1;
  while (t * kPer < experts) t *= 2;
  return t;
}

int64_t blocks_for(int64_t rows, int experts, int64_t most) {
  const int64_t per = kThreads / threads_of_row(experts), blocks = (rows + per - 1) / per;
  return blocks < most ? blocks : most;
}

template <typename T, int TPR>
void launch(const RouteArgs& a, unsigned blocks, hipStream_t stream) {
  hipLaunchKernelGGL(HIP_KERNEL_NAME(route_kernel<T, TPR>), dim3(blocks), dim3(kThreads), 0, stream, a);
}
template <typename T, int TPR>
void launch(const RouteGradArgs& a, unsigned blocks, hipStream_t stream) {
  hipLaunchKernelGGL(HIP_KERNEL_NAME(route_grad_kernel<T, TPR>), dim3(blocks), dim3(kThreads), 0, stream, a);
}
template <typename T, typename Args>
void launch_for(const Args& a, unsigned blocks, hipStream_t stream) {
  switch (threads_of_row(a.experts)) {
    case 1: return launch<T, 1>(a, blocks, stream);
    case 2: return launch<T, 2>(a, blocks, stream);
    case 4: return launch<T, 4>(a, blocks, stream);
    case 8: return launch<T, 8>(a, blocks, stream);
    case 16: return launch<T, 16>(a, blocks, stream);
    case 32: return launch<T, 32>(a, blocks, stream);
    default: return launch<T, 64>(a, blocks, stream);
  }
}
template <typename Args>
void launch_of(int dtype, const Args& a, unsigned blocks, hipStream_t stream) {
  if (dtype == DS_ELEM_F32) launch_for<float>(a, blocks, stream);
  else if (dtype == DS_ELEM_BF16) launch_for<__bf16>(a, blocks, stream);
  else launch_for<_Float16>(a, blocks, stream);
}

constexpr int64_t kMostBlocks = 512;   // that leave sums

}  // namespace

int64_t ds_route_bytes(int64_t rows, int experts) { return blocks_for(rows, experts, kMostBlocks) * (2 * (int64_t)experts + 1) * 4; }

int ds_launch_route(ds_ctx* ctx, int dtype, int64_t rows, int experts, int k, int renorm, ds_rows x, int32_t* ids, float* weights, int64_t* counts, float* loss,
                    float* lse, void* workspace) {
  const int64_t blocks = blocks_for(rows, experts, kMostBlocks);
  RouteArgs a = {};
  a.rows = rows;
  a.experts = experts;
  a.k = k;
  a.renorm = renorm != 0;
  a.x = x.data;
  a.xs = x.stride;
  a.ids = ids;
  a.weights = weights;
  a.counts = counts;
  a.loss = loss;
  a.lse = lse;
  a.sums = (float*)workspace;
  a.chosen = (int32_t*)workspace + blocks * experts;
  a.with = (int32_t*)workspace + 2 * blocks * experts;
  if (rows > 0) launch_of(dtype, a, (unsigned)blocks, ctx->stream);
  hipLaunchKernelGGL(route_join_kernel, dim3(1), dim3(1024), 0, ctx->stream, a, (int)blocks);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

int ds_launch_route_backward(ds_ctx* ctx, int dtype, int64_t rows, int experts, int k, int renorm, ds_rows x, const float* lse, const int32_t* ids,
                             const int64_t* counts, const float* dweights, const float* dloss, ds_rows dx) {
  if (rows == 0) return DS_OK;
  RouteGradArgs a = {};
  a.rows = rows;
  a.experts = experts;
  a.k = k;
  a.renorm = renorm != 0;
  a.x = x.data;
  a.xs = x.stride;
  a.lse = lse;
  a.ids = ids;
  a.counts = counts;
  a.dweights = dweights;
  a.dloss = dloss;
  a.dx = (void*)dx.data;
  a.ys = dx.stride;
  launch_of(dtype, a, (unsigned)blocks_for(rows, experts, 8 * (int64_t)ctx->num_cus), ctx->stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}
