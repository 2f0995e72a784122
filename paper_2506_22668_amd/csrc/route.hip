// The router's sums over all rows, and which kernels a call takes (route.h has them, a file for each type compiles them).
#include "route.h"

namespace {

// What the workgroups left, in order: 16 experts to a workgroup, 64 threads to an expert; the last workgroup that is through adds up their parts of the loss.
// Bound by latency: 64 experts of 512 workgroups 6.3 us.
constexpr int kJoinThreads = 1024, kJoinExperts = 16, kJoinParts = kJoinThreads / kJoinExperts;
__global__ __launch_bounds__(kJoinThreads) void route_join_kernel(RouteArgs a, int blocks) {
  __shared__ double sum_of[kJoinParts / 4][kJoinExperts];
  __shared__ int64_t number_of[kJoinParts / 4][kJoinExperts];
  __shared__ int turn;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = threadIdx.x / kJoinExperts, e = (int)blockIdx.x * kJoinExperts + lane % kJoinExperts;
  double s = 0.0;
  int64_t n = 0;
  if (e < a.experts) {
#pragma unroll 8
    for (int b = part; b < blocks; b += kJoinParts) {
      const float2 v = a.sums[(int64_t)b * a.experts + e];
      s += v.x;
      n += __float_as_int(v.y);
    }
  }
#pragma unroll
  for (int o = kJoinExperts; o < 64; o <<= 1) {
    s += __shfl_xor(s, o, 64);
    n += __shfl_xor(n, o, 64);
  }
  if (lane < kJoinExperts) {
    sum_of[wave][lane] = s;
    number_of[wave][lane] = n;
  }
  __syncthreads();
  if (wave > 0) return;
  s = 0.0;
  n = 0;
  if (lane < kJoinExperts) {
#pragma unroll
    for (int p = 0; p < kJoinParts / 4; ++p) {
      s += sum_of[p][lane];
      n += number_of[p][lane];
    }
  }
  if (lane < kJoinExperts && e < a.experts) a.counts[e] = n;
  double loss = s * (double)n;
  int64_t with = 0;
#pragma unroll 4
  for (int b = lane; b < blocks; b += 64) with += a.with[b];
  const auto add_up = [&]() {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      loss += __shfl_xor(loss, o, 64);
      n += __shfl_xor(n, o, 64);
    }
  };
  add_up();
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) with += __shfl_xor(with, o, 64);
  if (gridDim.x > 1) {   // (at most 64 workgroups: 1,024 experts)
    if (lane == 0) {
      a.losses[blockIdx.x] = loss;
      a.numbers[blockIdx.x] = n;
      __threadfence();
      turn = atomicAdd(a.through, 1);
    }
    if (__builtin_amdgcn_readfirstlane(turn) != (int)gridDim.x - 1) return;
    __threadfence();
    const bool there = lane < (int)gridDim.x;
    loss = there ? __hip_atomic_load(&a.losses[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    n = there ? __hip_atomic_load(&a.numbers[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    add_up();
  }
  if (lane == 0) {
    a.counts[a.experts] = with;
    *a.loss = (float)(loss * a.experts / ((double)(n > 0 ? n : 1) * (double)(with > 0 ? with : 1)));
  }
}

// Workgroups that leave sums: two to a compute unit. One takes up to two rounds of rows by itself, and nothing is left to add up.
constexpr int64_t kMostBlocks = 512, kAlone = 2;
int64_t sum_blocks(int64_t rows, int experts, bool f32) {
  const int64_t b = blocks_for(rows, experts, f32, kThreads, kMostBlocks);
  return b <= kAlone ? 1 : b;
}
int join_blocks(int experts) { return (experts + kJoinExperts - 1) / kJoinExperts; }

}  // namespace

// (of the type that has more workgroups)
int64_t ds_route_bytes(int64_t rows, int experts) {
  const int64_t a = sum_blocks(rows, experts, true), b = sum_blocks(rows, experts, false), blocks = a > b ? a : b;
  return blocks > 1 ? join_blocks(experts) * 16 + blocks * (2 * (int64_t)experts + 1) * 4 + 4 : 0;
}

int ds_launch_route(ds_ctx* ctx, int dtype, int64_t rows, int experts, int k, int renorm, ds_rows x, int32_t* ids, float* weights, int64_t* counts, float* loss,
                    float* lse, void* workspace) {
  const int64_t blocks = sum_blocks(rows, experts, dtype == DS_ELEM_F32);
  const int joins = join_blocks(experts);
  RouteArgs a = {};
  a.rows = rows;
  a.experts = experts;
  a.k = k;
  a.renorm = renorm != 0;
  a.low = experts > 1 ? (2u << (31 - __builtin_clz((unsigned)experts - 1))) - 1 : 1;
  a.x = x.data;
  a.xs = x.stride;
  a.ids = ids;
  a.weights = weights;
  a.counts = counts;
  a.loss = loss;
  a.lse = lse;
  a.losses = (double*)workspace;
  a.numbers = (int64_t*)workspace + joins;
  a.sums = (float2*)workspace + 2 * joins;
  a.with = (int32_t*)(a.sums + blocks * experts);
  a.through = a.with + blocks;
  const unsigned grid = (unsigned)blocks;
  if (dtype == DS_ELEM_F32) ds_route_rows<float>(&a, grid, ctx->stream);
  else if (dtype == DS_ELEM_BF16) ds_route_rows<__bf16>(&a, grid, ctx->stream);
  else ds_route_rows<_Float16>(&a, grid, ctx->stream);
  if (blocks > 1) hipLaunchKernelGGL(route_join_kernel, dim3(joins), dim3(kJoinThreads), 0, ctx->stream, a, (int)blocks);
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
  const unsigned grid = (unsigned)blocks_for(rows, experts, dtype == DS_ELEM_F32, kGradThreads, 4 * (int64_t)ctx->num_cus);
  if (dtype == DS_ELEM_F32) ds_route_rows_backward<float>(&a, grid, ctx->stream);
  else if (dtype == DS_ELEM_BF16) ds_route_rows_backward<__bf16>(&a, grid, ctx->stream);
  else ds_route_rows_backward<_Float16>(&a, grid, ctx->stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}
