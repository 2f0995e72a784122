// Rows by group: offsets[g] rows lie in the groups before g, and the order lists the rows group by group, ascending within a
// group, those of no group (an id outside of [0, groups)) last.
//
// A stable counting sort with one key digit. A workgroup of 16 waves has a stretch of the rows, every wave a sixteenth of it in
// steps of 64. Within a step the lanes of one group find each other by a ballot for every bit of the id, so that a row's rank is
// a popcount and the lowest lane adds the step's count in LDS: no atomic decides an order, and the result is the
// only one there is. Several workgroups: a first launch leaves every stretch's counts, a second adds up the ones before its own
// (ids are read twice, from the caches the second time). Its bytes are nothing (1,000,175 rows 1.6 us): what it takes is the latency of its steps.
// 1,010 rows in 8 groups 8 us; 1,000,175 rows in 64 groups 19 us (counts 6, places 14, of which every workgroup's reading of all counts is 5);
// 10,000,000 rows in 64 groups 137 us. Where the counts are many, a launch between the two adds them up.
#include "feature_ops.h"
#include "rows.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kStretch = 2048;    // rows of a workgroup, at the least, where there are several (12,000 rows in 64 groups: 4,096 22.6 us, 2,048 11.7)

constexpr int kMostBlocks = 256;   // workgroups (one to a compute unit: their counts in LDS)
constexpr int kSummed = 28000;     // counts from which a launch of its own adds them up, below which every workgroup does (1,000,175 rows in 64 groups,
                                   // 16,640 counts: 21.5 us with the launch, 19.3 without; 100,000 in 1,000, 49,049: 17.0, 22.2; 1,000,000 in 1,024: 29, 63)

struct GroupArgs {
  const int32_t* ids;
  int rows, groups, per_wave;   // rows of a wave, a multiple of 64
  int64_t* offsets;
  int32_t *order, *counts;      // counts: [block][groups + 1], and behind them the groups' rows
  bool summed;                  // group_before_kernel has been over the counts
};

// the lanes whose key is this lane's
__device__ __forceinline__ unsigned long long same_key(int key, int bits) {
  unsigned long long same = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const unsigned long long set = __ballot((key >> b) & 1);
    same &= (key >> b) & 1 ? set : ~set;
  }
  return same;
}

__device__ __forceinline__ int key_of(const GroupArgs& a, int row, int end) {
  if (row >= end) return a.groups + 1;   // (counted nowhere)
  const int id = a.ids[row];
  return id >= 0 && id < a.groups ? id : a.groups;
}

// Goes through a wave's rows: calls each(row, key, rank among the step's rows of the key, how many) for the rows there are
template <typename Each>
__device__ __forceinline__ void walk(const GroupArgs& a, int wave, Each each) {
  const int lane = threadIdx.x & 63, bits = 32 - __clz(a.groups + 1);
  const int64_t first = ((int64_t)blockIdx.x * kWaves + wave) * a.per_wave;
  const int begin = first < a.rows ? (int)first : a.rows;
  const int end = a.rows - begin < a.per_wave ? a.rows : begin + a.per_wave;
  // (the ids of four steps are on their way at a time, those of the next four while these are worked off)
  int next[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) next[j] = key_of(a, begin + j * 64 + lane, end);
  for (int at = begin; at < end; at += 256) {
    int now[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      now[j] = next[j];
      next[j] = end - at > 256 ? key_of(a, at + 256 + j * 64 + lane, end) : 0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (end - at <= j * 64) break;
      const unsigned long long same = same_key(now[j], bits);
      const int rank = __popcll(same & ((1ull << lane) - 1));
      each(at + j * 64 + lane, now[j], rank, __popcll(same));
    }
  }
}

// counts of this workgroup's rows by wave and group
__device__ __forceinline__ void count_rows(const GroupArgs& a, int* count) {
  const int wave = threadIdx.x >> 6, keys = a.groups + 1;
  for (int i = threadIdx.x; i < kWaves * keys; i += kThreads) count[i] = 0;
  __syncthreads();
  volatile int* mine = count + wave * keys;   // (lanes of the wave take turns at it)
  walk(a, wave, [&](int, int key, int rank, int of) {
    if (rank == 0 && key < keys) mine[key] = mine[key] + of;   // (one lane a group)
  });
  __syncthreads();
}

__global__ __launch_bounds__(kThreads) void group_count_kernel(GroupArgs a) {
  extern __shared__ int count[];
  count_rows(a, count);
  const int keys = a.groups + 1;
  for (int g = threadIdx.x; g < keys; g += kThreads) {
    int n = 0;
    for (int w = 0; w < kWaves; ++w) n += count[w * keys + g];
    a.counts[(int64_t)blockIdx.x * keys + g] = n;
  }
}

// Turns the workgroups' counts into the rows of the group before each of them, and leaves the groups' rows behind them: a lane a group, every wave a
// sixteenth of the (at most 256) workgroups
__global__ __launch_bounds__(kThreads) void group_before_kernel(GroupArgs a, int blocks) {
  __shared__ int sum[kWaves][64];
  const int keys = a.groups + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, key = (int)blockIdx.x * 64 + lane;
  const int each = (blocks + kWaves - 1) / kWaves, first = wave * each;
  int n[kMostBlocks / kWaves], all = 0;
#pragma unroll
  for (int j = 0; j < kMostBlocks / kWaves; ++j)
    n[j] = j < each && first + j < blocks && key < keys ? a.counts[(int64_t)(first + j) * keys + key] : 0;
#pragma unroll
  for (int j = 0; j < kMostBlocks / kWaves; ++j) all += n[j];
  sum[wave][lane] = all;
  __syncthreads();
  int before = 0, whole = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sum[w][lane];
    whole += sum[w][lane];
  }
  if (key >= keys) return;
#pragma unroll
  for (int j = 0; j < kMostBlocks / kWaves; ++j) {
    if (j < each && first + j < blocks) a.counts[(int64_t)(first + j) * keys + key] = before;
    before += n[j];
  }
  if (wave == 0) a.counts[(int64_t)blocks * keys + key] = whole;
}

__global__ __launch_bounds__(kThreads) void group_place_kernel(GroupArgs a) {
  extern __shared__ int count[];   // [waves][keys], then the rows of a group in the whole and before this workgroup
  __shared__ int wave_sum[kWaves];
  const int keys = a.groups + 1, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int *whole = count + kWaves * keys, *before = whole + keys;
  count_rows(a, count);
  if (gridDim.x == 1) {
    for (int g = threadIdx.x; g < keys; g += kThreads) {
      int n = 0;
      for (int w = 0; w < kWaves; ++w) n += count[w * keys + g];
      whole[g] = n;
      before[g] = 0;
    }
  } else if (a.summed) {
    const int mine = (int)blockIdx.x * keys, all = (int)gridDim.x * keys;
    for (int g = threadIdx.x; g < keys; g += kThreads) {
      before[g] = a.counts[mine + g];
      whole[g] = a.counts[all + g];
    }
  } else {
    for (int g = threadIdx.x; g < keys; g += kThreads) whole[g] = before[g] = 0;
    __syncthreads();
    // eight counts a thread at a time: each is a load of its own from the caches (one at a time: 17 us of 1,000,175 rows in 64 groups)
    const int all = (int)gridDim.x * keys, mine = (int)blockIdx.x * keys;
    for (int base = threadIdx.x; base < all; base += 8 * kThreads) {
      int n[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) n[j] = base + j * kThreads < all ? a.counts[base + j * kThreads] : 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (n[j] == 0) continue;
        const int i = base + j * kThreads, g = i % keys;
        atomicAdd(&whole[g], n[j]);   // (whole numbers: any order gives the same)
        if (i < mine) atomicAdd(&before[g], n[j]);
      }
    }
  }
  __syncthreads();
  // where each group starts
  const int n = (int)threadIdx.x < a.groups ? whole[threadIdx.x] : 0;
  int upto = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o, 64);
    if (lane >= o) upto += up;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  int start = upto - n, held = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) start += wave_sum[w];
    held += wave_sum[w];
  }
  for (int g = threadIdx.x; g < keys; g += kThreads) {
    // (thread g has group g's start; the rows of no group start behind all others)
    int at = (g < a.groups ? start : held) + before[g];
    if (blockIdx.x == 0) a.offsets[g] = at;
    for (int w = 0; w < kWaves; ++w) {
      const int c = count[w * keys + g];
      count[w * keys + g] = at;
      at += c;
    }
  }
  __syncthreads();
  volatile int* mine = count + wave * keys;
  walk(a, wave, [&](int row, int key, int rank, int of) {
    if (key >= keys) return;
    const int at = mine[key];
    a.order[at + rank] = row;
    if (rank == 0) mine[key] = at + of;   // (a wave's LDS accesses keep their order)
  });
}

}  // namespace

// One workgroup takes up to four stretches by itself: a second launch costs more than the rest of its walk does (6,000 rows in 64 groups: 12.0 us in
// one, 14.2 in two; 8,000: 15.1, 14.0, in 4 groups 11.3, 13.9).
int ds_group_blocks(int rows) {
  const int blocks = (rows + kStretch - 1) / kStretch;
  return blocks <= 4 ? 1 : blocks < kMostBlocks ? blocks : kMostBlocks;
}

int ds_launch_group_rows(ds_ctx* ctx, const int32_t* ids, int rows, int groups, int64_t* offsets, int32_t* order, int32_t* counts) {
  const int blocks = ds_group_blocks(rows);
  GroupArgs a = {};
  a.ids = ids;
  a.rows = rows;
  a.groups = groups;
  const int64_t waves = (int64_t)blocks * kWaves, each = ((int64_t)rows + waves - 1) / waves;
  a.per_wave = (int)((each + 63) / 64 * 64);
  a.offsets = offsets;
  a.order = order;
  a.counts = counts;
  const int lds = (kWaves + 2) * (groups + 1) * (int)sizeof(int);
  if (lds > 48 * 1024) {
    DS_HIP(ctx, hipFuncSetAttribute((const void*)group_count_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    DS_HIP(ctx, hipFuncSetAttribute((const void*)group_place_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  }
  if (blocks > 1) hipLaunchKernelGGL(group_count_kernel, dim3(blocks), dim3(kThreads), lds, ctx->stream, a);
  a.summed = blocks > 1 && blocks * (groups + 1) >= kSummed;
  if (a.summed) hipLaunchKernelGGL(group_before_kernel, dim3((groups + 64) / 64), dim3(kThreads), 0, ctx->stream, a, blocks);
  hipLaunchKernelGGL(group_place_kernel, dim3(blocks > 0 ? blocks : 1), dim3(kThreads), lds, ctx->stream, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}
