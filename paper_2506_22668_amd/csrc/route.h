// The experts of every row from a router's scores, how evenly they are used, and the scores' gradient.
//
//   forward:   p = softmax(x) over a row's experts; ids: those of the k highest scores, ties to the lowest, -inf never; w_j = p at id_j, or its share of
//              the k; counts_e = how often e was chosen, N = rows with an expert; loss = E sum_e (counts_e / sum of counts) (sum_r p_re / N)
//   backward:  dx = p (g - sum_e p g), g_e = dloss E counts_e / (N sum of counts) + [e = id_j] dp_j,
//              dp_j = dw_j, or (dw_j - sum_i dw_i w_i) / sum of the chosen p
//
// A row of up to 1,024 scores stays in the registers of TPR threads, PER to a thread. A row that is -inf throughout has no expert: ids -1, weights 0, and it takes no
// part in N. One with NaN or +inf has none either, but its weights, and so the loss, are NaN. All sums are fp32, over rows first in a thread, then in
// a workgroup, and the workgroups' in 64 bits in a fixed order: the same inputs give the same bits.
//
// Vector instructions, not memory, are what such a kernel runs out of first (a wave's take four cycles: 1,000,175 rows of 64 bf16 in 29 us leave 18 a score), so:
//  - a score and its expert are one integer, ordered as scores are and, of equal ones, the lowest expert first: a thread's k highest are a list that each
//    score passes through in one median and one maximum of three a place, and the row's are the threads' heads, highest first. A 16-bit score
//    leaves 13 bits of 32 free for the expert. Of an fp32 one the last bits give way to it, which orders all scores but those that differ in these bits alone:
//    a list of k + 1 shows where that is so, and these rows are gone through again, k times, in full.
//  - e^(x - top) is one exponential of base 2, of x log2(e) - top log2(e) in one fused product where a row's highest score is below 2^16 (beyond, what the second term
//    is rounded by would count: there the difference is formed first). It knows no subnormal results; where they matter, it is squared from half the power.
#pragma once
#include <math.h>

#include <type_traits>

#include "feature_ops.h"
#include "rows.h"

namespace {

constexpr float kLog2e = 1.44269504088896341f, kHalf = 0.5f * kLog2e, kLn2 = 0.693147180559945309f;

struct RouteArgs {
  int64_t rows;
  int experts, k;
  bool renorm;
  uint32_t low;         // the bits of a key that hold the expert
  const void* x;
  int64_t xs;
  int32_t* ids;
  float *weights, *loss, *lse;
  int64_t* counts;
  // what workgroups leave, where there are several: sums of p and counts [block][experts], rows [block]; and of the workgroups that add these up,
  // their part of the loss and of the counts, and how many are through
  float2* sums;
  int32_t *with, *through;
  double* losses;
  int64_t* numbers;
};

template <int CTRL>
__device__ __forceinline__ int across(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
// The highest of LANES neighbouring lanes, in each of them
template <int LANES>
__device__ __forceinline__ int max_lanes(int v) {
  if constexpr (LANES >= 2) v = max(v, across<0xB1>(v));
  if constexpr (LANES >= 4) v = max(v, across<0x4E>(v));
  if constexpr (LANES >= 8) v = max(v, across<0x141>(v));
  if constexpr (LANES >= 16) v = max(v, across<0x140>(v));
  if constexpr (LANES >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = max((int)p[0], (int)p[1]);
  }
  if constexpr (LANES >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    v = max((int)p[0], (int)p[1]);
  }
  return v;
}

template <int LANES>
__device__ __forceinline__ float highest_lane(float v) {
  if constexpr (LANES >= 2) v = fmaxf(v, __int_as_float(across<0xB1>(__float_as_int(v))));
  if constexpr (LANES >= 4) v = fmaxf(v, __int_as_float(across<0x4E>(__float_as_int(v))));
  if constexpr (LANES >= 8) v = fmaxf(v, __int_as_float(across<0x141>(__float_as_int(v))));
  if constexpr (LANES >= 16) v = fmaxf(v, __int_as_float(across<0x140>(__float_as_int(v))));
  if constexpr (LANES >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  if constexpr (LANES >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  return v;
}

// e^d; 0 below 2^-126
__device__ __forceinline__ float power_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
// 2^(2 d) with subnormal results
__device__ __forceinline__ float squared_power(float d) {
  const float e = __builtin_amdgcn_exp2f(d);
  return e * e;
}
__device__ __forceinline__ float whole_power(float d) { return squared_power(0.5f * d); }

// Element `row` (of up to 2^30, each of four bytes) behind an address that all lanes share
template <typename V>
__device__ __forceinline__ V& at_row(V* base, uint32_t row) {
  return *reinterpret_cast<V*>(reinterpret_cast<char*>(const_cast<typename std::remove_const<V>::type*>(base)) + row * 4u);
}

// A thread's scores: pieces of 16 bytes, a row's threads side by side; `absent` where the row has ended
template <typename T, int TPR, int PER>
struct Scores {
  static constexpr int N = Piece<T>::N, PIECES = PER / N;
  PieceV<T> v[PIECES];
  __device__ __forceinline__ void load(const T* row, int t, int experts) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (p * TPR + t) * N;
      if (experts < N) v[p] = load_piece<T>(row + at, experts - at);
      else v[p] = *reinterpret_cast<const typename Piece<T>::U*>(row + min(at, experts - N));
    }
  }
  __device__ __forceinline__ void read(int t, int experts, float absent, float (&to)[PER]) {
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (p * TPR + t) * N, have = experts - at;
      if (have >= N) {
#pragma unroll
        for (int i = 0; i < N; ++i) to[p * N + i] = (float)v[p][i];
      } else {
        if (experts >= N && have > 0) v[p] = shifted<T>(v[p], (unsigned)(N - have));
#pragma unroll
        for (int i = 0; i < N; ++i) to[p * N + i] = i < have ? (float)v[p][i] : absent;
      }
    }
  }
};
// the expert of a thread's score i
template <typename T, int TPR>
__device__ __forceinline__ int expert_of(int t, int i) {
  constexpr int N = Piece<T>::N;
  return (i / N * TPR + t) * N + i % N;
}

// A score's key, less the expert: ordered as whole numbers as the scores are (-0 as 0), `low` bits cleared
__device__ __forceinline__ uint32_t key_of(float v, uint32_t low) {
  const uint32_t bits = __float_as_uint(v + 0.f);
  return (bits ^ ((uint32_t)((int)bits >> 31) & (0x7fffffffu & ~low))) & ~low;
}
__device__ __forceinline__ float score_of(int key, uint32_t low) {
  const uint32_t t = (uint32_t)key & ~low;
  return __uint_as_float(t ^ ((uint32_t)((int)t >> 31) & (0x7fffffffu & ~low)));
}

// The highest K of a thread's keys, highest first
template <int K, int PER>
__device__ __forceinline__ void highest(const int (&key)[PER], int (&list)[K]) {
#pragma unroll
  for (int i = 0; i < PER; ++i) {
#pragma unroll
    for (int j = K - 1; j > 0; --j) asm("v_med3_i32 %0, %1, %2, %0" : "+v"(list[j]) : "v"(list[j - 1]), "v"(key[i]));   // (the compiler makes two of it)
    list[0] = max(list[0], key[i]);
  }
}

// Counts of a row's experts are added up in LDS (whole numbers: in any order). Bound by vector instructions: 1,000,175 rows of 64 bf16, 2 of them each, 38.5 us, about 18 a score (29 for the
// bytes); 30,011 rows of 515 fp32, 8 of them each, 40.1 (12.6 for the bytes). Of the latter a row, a wave, takes about 600: the list of nine places 80, the
// eight further picks 190, with some 50 waits between dependent steps across lanes, and a third of the places of all threads but one hold no score. 16-bit rows
// whose experts do not fill the places of a power of two of threads are farthest from their bytes: of 2^25 scores, k 1, 33, 300 and 515 experts 47, 39 and 41 us, 64,
// 256 and 1,024 28, 28 and 27.
template <typename T, int TPR, int PER, int K, int THREADS>
__global__ __launch_bounds__(THREADS) void route_kernel(RouteArgs a) {
  constexpr int ROWS = THREADS / TPR, WAVES = THREADS / 64, WIDE = TPR * PER, LIST = sizeof(T) == 4 ? K + 1 : K, OWN = (K + TPR - 1) / TPR;
  // the waves' sums, at the end; until then, fp32: the scores of the rows under way, from which those that were chosen are read
  __shared__ __attribute__((aligned(16))) float room[sizeof(T) == 4 ? THREADS * PER : WAVES * WIDE];
  float* mine = room + (int)threadIdx.x / TPR * WIDE;
  __shared__ int count[WIDE], with_of[WAVES];
  const int t = threadIdx.x % TPR;
  const float none = -INFINITY;
  const int lowest = (int)(0x80000000u), shut = (int)(key_of(none, a.low) | a.low);   // at or below: -inf, or no score
  for (int e = threadIdx.x; e < WIDE; e += THREADS) count[e] = 0;
  __syncthreads();
  const uint32_t step = gridDim.x * ROWS, rows = (uint32_t)a.rows;   // (at most 2^30)
  uint32_t row = blockIdx.x * ROWS + threadIdx.x / TPR;
  float sum[PER] = {};
  int with = 0;
  Scores<T, TPR, PER> next = {};
  if (row < rows) next.load((const T*)a.x + row * a.xs, t, a.experts);
  for (; row < rows; row += step) {
    Scores<T, TPR, PER> now = next;
    if (row + step < rows) next.load((const T*)a.x + (row + step) * a.xs, t, a.experts);
    float x[PER];
    now.read(t, a.experts, none, x);
    int list[LIST];
    {
      int key[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        // (where the row has ended the score is -inf, and which expert its key names does not matter)
        key[i] = (int)(key_of(x[i], a.low) | ((a.low - (uint32_t)expert_of<T, TPR>(t, i)) & a.low));
      }
#pragma unroll
      for (int j = 0; j < LIST; ++j) list[j] = lowest;
      highest(key, list);
    }
    // (thread t of the row has its choices t, t + TPR, ..)
    int own[OWN], first = lowest, last = lowest;
    bool again = false;   // fp32: scores that are told apart by their last bits alone
#pragma unroll
    for (int c = 0; c < OWN; ++c) own[c] = lowest;
#pragma unroll
    for (int j = 0; j < LIST; ++j) {
      if (j >= a.k + (LIST - K)) continue;
      const int best = max_lanes<TPR>(list[0]);
      if constexpr (sizeof(T) == 4) again |= j > 0 && best > shut && ((best ^ last) & ~a.low) == 0;
      last = best;
      if (j == 0) first = best;
      if (j < K && j < a.k) own[j < K ? j / TPR : 0] = t == j % TPR ? best : own[j < K ? j / TPR : 0];
      if (list[0] == best) {   // (of what comes behind the last K - j nothing is asked for any more)
#pragma unroll
        for (int i = 0; i + 1 < LIST - j; ++i) list[i] = list[i + 1];
      }
    }
    float top = first > shut ? score_of(first, a.low) : 0.f;
    if constexpr (sizeof(T) == 4) {   // (a key's bits alone may be far from a large score)
      top = none;
      __builtin_amdgcn_wave_barrier();   // (a row's threads are of one wave, whose LDS accesses keep their order)
#pragma unroll
      for (int p = 0; p < PER / 4; ++p) *reinterpret_cast<float4*>(mine + (p * TPR + t) * 4) = float4{x[4 * p], x[4 * p + 1], x[4 * p + 2], x[4 * p + 3]};
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int i = 0; i < PER; ++i) top = fmaxf(top, x[i]);
      top = highest_lane<TPR>(top);
      if (top == none) top = 0.f;
    }
    float q[PER], total = 0.f;
    // (the second term's rounding is the same for a whole row, so it cancels in p; `shift` is the power that the highest score itself gets by it, exactly, and lse goes without it)
    const bool near = fabsf(top) < 65536.f;
    const float base = top * kLog2e, shift = near ? fmaf(top, kLog2e, -base) : 0.f;
    if (near) {
#pragma unroll
      for (int i = 0; i < PER; ++i) q[i] = __builtin_amdgcn_exp2f(fmaf(x[i], kLog2e, -base));
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) q[i] = power_of(x[i] - top);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) total += q[i];
    total = sum_lanes<TPR>(total);
    const bool fine = total > 0.f && total < INFINITY;   // (a NaN is neither; a row without an open expert sums up to 0)
    const float inv = total == 0.f ? 0.f : __builtin_amdgcn_rcpf(total);
#pragma unroll
    for (int i = 0; i < PER; ++i) sum[i] = fmaf(q[i], inv, sum[i]);
    with += fine && t == 0;
    int exact[OWN] = {};
    if (sizeof(T) == 4 && __any(again)) {
#pragma clang loop unroll(disable)
      for (int j = 0; j < a.k; ++j) {
        float best = none;
        int at = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const bool above = x[i] > best;
          best = above ? x[i] : best;
          at = above ? expert_of<T, TPR>(t, i) : at;
        }
        const float most = highest_lane<TPR>(best);
        const int lowest_expert = -max_lanes<TPR>(best == most ? -at : -0x7fffffff), found = most > none ? lowest_expert : -1;
#pragma unroll
        for (int c = 0; c < OWN; ++c) exact[c] = j == c * TPR + t ? found : exact[c];
#pragma unroll
        for (int i = 0; i < PER; ++i) x[i] = expert_of<T, TPR>(t, i) == found ? none : x[i];
      }
    }
    int id[OWN];
    float weight[OWN], shares = 0.f;
#pragma unroll
    for (int c = 0; c < OWN; ++c) {
      id[c] = fine && own[c] > shut ? (int)(a.low - ((uint32_t)own[c] & a.low)) : -1;
      if (sizeof(T) == 4 && again && fine) id[c] = exact[c];
      float score;
      if constexpr (sizeof(T) == 4) score = id[c] < 0 ? none : mine[id[c]];
      else score = score_of(own[c], a.low);
      weight[c] = id[c] >= 0 ? whole_power(near ? fmaf(score, kLog2e, -base) : (score - top) * kLog2e) * inv : fine || total == 0.f ? 0.f : NAN;
      shares += sum_lanes<TPR>(c * TPR + t < a.k ? weight[c] : 0.f);
    }
    const float by = a.renorm && shares > 0.f ? __builtin_amdgcn_rcpf(shares) : 1.f;
#pragma unroll
    for (int c = 0; c < OWN; ++c) {
      const int j = c * TPR + t;
      if (j < a.k) {
        const int64_t at = j * a.rows + row;
        a.ids[at] = id[c];
        a.weights[at] = weight[c] * by;
        if (id[c] >= 0) atomicAdd(&count[id[c]], 1);
      }
    }
    if (t == 0 && a.lse) at_row(a.lse, row) = total == 0.f ? none : fmaf(__log2f(total) - shift, kLn2, top);
  }
  if constexpr (sizeof(T) == 4) __syncthreads();
  // the workgroup's rows: those of a wave first (lanes TPR apart)
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
#pragma unroll
    for (int o = TPR; o < 64; o <<= 1) sum[i] += __shfl_xor(sum[i], o, 64);
    if (lane < TPR) room[wave * WIDE + expert_of<T, TPR>(t, i)] = sum[i];
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) with += __shfl_xor(with, o, 64);
  if (lane == 0) with_of[wave] = with;
  __syncthreads();
  const bool alone = gridDim.x == 1;
  double loss = 0.0;
  int number = 0;
  for (int e = threadIdx.x; e < a.experts; e += THREADS) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += room[w * WIDE + e];
    if (alone) {
      a.counts[e] = count[e];
      loss += (double)s * count[e];
      number += count[e];
    } else {
      a.sums[(int64_t)blockIdx.x * a.experts + e] = float2{s, __int_as_float(count[e])};
    }
  }
  int all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) all += with_of[w];
  if (!alone) {
    if (threadIdx.x == 0) {
      a.with[blockIdx.x] = all;
      if (blockIdx.x == 0) *a.through = 0;
    }
    return;
  }
  __syncthreads();
  double* part = reinterpret_cast<double*>(room);
  static_assert(sizeof(room) >= 16 * WAVES, "");
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    loss += __shfl_xor(loss, o, 64);
    number += __shfl_xor(number, o, 64);
  }
  if (lane == 0) {
    part[wave] = loss;
    part[WAVES + wave] = (double)number;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    double sum_loss = 0.0, chosen = 0.0;
    for (int w = 0; w < WAVES; ++w) {
      sum_loss += part[w];
      chosen += part[WAVES + w];
    }
    a.counts[a.experts] = all;
    // (a sum that is NaN stays one, where nothing was chosen too)
    *a.loss = (float)(sum_loss * a.experts / (fmax(chosen, 1.0) * (double)(all > 0 ? all : 1)));
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

// The scores that were chosen are read once more, each by its address: a row's sum takes their gradients from there, and the threads that hold them take them from a row
// in LDS, which is zero but for them (comparing experts in the registers takes four instructions a score and choice). Only the row's own threads, of one
// wave, touch it, and a wave's LDS accesses keep their order. What e^(x - lse) is off by lse's own rounding, which grows with the scores (1,000: 3e-5; where all are the type's
// lowest value lse is that value, and each power 1), is the same for a row's experts: their sum takes it out. Bound by memory: 131,072 rows of 256 bf16, 4 of them each, 28.2 us, 4.9 TB/s.
template <typename T, int TPR, int PER, int K, int THREADS>
__global__ __launch_bounds__(THREADS) void route_grad_kernel(RouteGradArgs a) {
  constexpr int ROWS = THREADS / TPR, N = Piece<T>::N, PIECES = PER / N, OWN = (K + TPR - 1) / TPR;
  __shared__ __attribute__((aligned(16))) float added[ROWS][TPR * PER];
  const int t = threadIdx.x % TPR;
  const float none = -INFINITY;
  float* mine = added[threadIdx.x / TPR];
  // the loss' part of g: the same for all rows
  float share[PER] = {};
  if (a.dloss) {
    // (every wave for itself: whole numbers below 2^53)
    double chosen = 0.0;
    for (int e = threadIdx.x & 63; e < a.experts; e += 64) chosen += (double)a.counts[e];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) chosen += __shfl_xor(chosen, o, 64);
    const int64_t with = a.counts[a.experts];
    const double by = (double)*a.dloss * a.experts / ((chosen > 0.0 ? chosen : 1.0) * (double)(with > 0 ? with : 1));
    static_assert(THREADS >= TPR, "a row of `added` holds every expert");
    float* all = &added[0][0];
    for (int e = threadIdx.x; e < TPR * PER; e += THREADS) all[e] = e < a.experts ? (float)(by * (double)a.counts[e]) : 0.f;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) share[i] = all[expert_of<T, TPR>(t, i)];
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) mine[expert_of<T, TPR>(t, i)] = 0.f;
  const uint32_t step = gridDim.x * ROWS, rows = (uint32_t)a.rows;   // (at most 2^30)
  uint32_t row = blockIdx.x * ROWS + threadIdx.x / TPR;
  // A row's scores, those that were chosen among them, come in while the row before is worked off; which ones were chosen, while the one before that is.
  Scores<T, TPR, PER> next = {};
  // (thread t of the row has its choices t, t + TPR, ..)
  int late_id[OWN] = {}, next_id[OWN];
  float late_dw[OWN] = {}, next_dw[OWN], late_lse = none, next_lse = none;
  T next_of[OWN];
  const auto look_up = [&](uint32_t r) __attribute__((always_inline)) {
    if (r >= rows) return;
    late_lse = at_row(a.lse, r);
    if (!a.dweights) return;
#pragma unroll
    for (int c = 0; c < OWN; ++c) {
      const int j = c * TPR + t;
      late_id[c] = -1;
      if (j < a.k) {
        late_id[c] = a.ids[j * a.rows + r];
        late_dw[c] = a.dweights[j * a.rows + r];
      }
    }
  };
  const auto fetch = [&](uint32_t r) __attribute__((always_inline)) {
    if (r >= rows) return;
    const T* from = (const T*)a.x + r * a.xs;
    next.load(from, t, a.experts);
    next_lse = late_lse;
    if (!a.dweights) return;
#pragma unroll
    for (int c = 0; c < OWN; ++c) {
      next_dw[c] = late_dw[c];
      next_id[c] = (uint32_t)late_id[c] < (uint32_t)a.experts ? late_id[c] : -1;
      next_of[c] = from[next_id[c] < 0 ? 0 : next_id[c]];
    }
  };
  look_up(row);
  fetch(row);
  look_up(row + step);
  for (; row < rows; row += step) {
    Scores<T, TPR, PER> now = next;
    int id[OWN];
    float dp[OWN], of[OWN];
    const float base = next_lse == none ? 0.f : next_lse;
#pragma unroll
    for (int c = 0; c < OWN; ++c) {
      id[c] = next_id[c];
      dp[c] = next_dw[c];
      of[c] = (float)next_of[c];
    }
    fetch(row + step);
    look_up(row + 2 * step);
    float p[PER], s = 0.f, own = 0.f, sum = 0.f;
    now.read(t, a.experts, none, p);
    // (the exponents of half the power, as in the forward pass, rounded alike for the whole row; a row that is closed throughout: 0)
    const bool near = fabsf(base) < 65536.f;
    const float half = base * kHalf;
    if (near) {
#pragma unroll
      for (int i = 0; i < PER; ++i) p[i] = squared_power(fmaf(p[i], kHalf, -half));
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) p[i] = squared_power((p[i] - base) * kHalf);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      sum += p[i];
      s = fmaf(p[i], share[i], s);
    }
    sum = sum_lanes<TPR>(sum);
    const float part = sum > 0.f ? __builtin_amdgcn_rcpf(sum) : 1.f;
    s = sum_lanes<TPR>(s) * part;
    float g[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) g[i] = share[i];
    if (a.dweights) {
      float dot = 0.f, total = 0.f;
#pragma unroll
      for (int c = 0; c < OWN; ++c) {
        of[c] = id[c] < 0 ? 0.f : squared_power(near ? fmaf(of[c], kHalf, -half) : (of[c] - base) * kHalf) * part;
        dp[c] = id[c] < 0 ? 0.f : dp[c];
        total += of[c];
        dot = fmaf(dp[c], of[c], dot);
      }
      total = sum_lanes<TPR>(total);
      dot = sum_lanes<TPR>(dot);
      const float inv = a.renorm ? total > 0.f ? __builtin_amdgcn_rcpf(total) : 0.f : 1.f;
      dot = a.renorm ? dot * inv : 0.f;
#pragma unroll
      for (int c = 0; c < OWN; ++c) {
        dp[c] = id[c] < 0 ? 0.f : (dp[c] - dot) * inv;
        own = fmaf(dp[c], of[c], own);
        if (id[c] >= 0) mine[id[c]] = dp[c];
      }
      own = sum_lanes<TPR>(own);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int q = 0; q < PIECES; ++q)
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const float4 v = *reinterpret_cast<const float4*>(mine + (q * TPR + t) * N + i);
          g[q * N + i] += v.x;
          g[q * N + i + 1] += v.y;
          g[q * N + i + 2] += v.z;
          g[q * N + i + 3] += v.w;
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int c = 0; c < OWN; ++c)
        if (id[c] >= 0) mine[id[c]] = 0.f;
      __builtin_amdgcn_wave_barrier();
    }
    s = (s + own) * part;
    T* dx = (T*)a.dx + row * a.ys;
#pragma unroll
    for (int q = 0; q < PIECES; ++q) {
      const int at = (q * TPR + t) * N;
      PieceV<T> out;
#pragma unroll
      for (int i = 0; i < N; ++i) out[i] = (T)(p[q * N + i] * fmaf(g[q * N + i], part, -s));
      store_piece<T>(dx + at, out, a.experts - at);
    }
  }
}

// Scores of a thread and threads of a row: 16, or 24 of 16 bits (12 of fp32) where that takes fewer places
struct Form {
  int per, threads;
};
inline Form form_of(int experts, bool f32) {
  if (experts <= 8) return {8, 1};
  int t = 1;
  while (t * 16 < experts) t *= 2;
  if (f32) return t * 12 >= experts ? Form{12, t} : Form{16, t};
  return t >= 2 && t / 2 * 24 >= experts ? Form{24, t / 2} : Form{16, t};
}

constexpr int kThreads = 512, kGradThreads = 256;
inline int64_t blocks_for(int64_t rows, int experts, bool f32, int threads, int64_t most) {
  const int64_t per = threads / form_of(experts, f32).threads, blocks = (rows + per - 1) / per;
  return blocks < most ? blocks : most;
}

template <typename T, int TPR, int PER, int K>
void launch(const RouteArgs& a, unsigned blocks, hipStream_t stream) {
  hipLaunchKernelGGL(HIP_KERNEL_NAME(route_kernel<T, TPR, PER, K, kThreads>), dim3(blocks), dim3(kThreads), 0, stream, a);
}
template <typename T, int TPR, int PER, int K>
void launch(const RouteGradArgs& a, unsigned blocks, hipStream_t stream) {
  hipLaunchKernelGGL(HIP_KERNEL_NAME(route_grad_kernel<T, TPR, PER, K, kGradThreads>), dim3(blocks), dim3(kGradThreads), 0, stream, a);
}
template <typename T, int TPR, int PER, typename Args>
void launch_k(const Args& a, unsigned blocks, hipStream_t stream) {
  if (a.k == 1) launch<T, TPR, PER, 1>(a, blocks, stream);
  else if (a.k == 2) launch<T, TPR, PER, 2>(a, blocks, stream);
  else if (a.k <= 4) launch<T, TPR, PER, 4>(a, blocks, stream);
  else launch<T, TPR, PER, 8>(a, blocks, stream);
}
template <typename T, typename Args>
void launch_for(const Args& a, unsigned blocks, hipStream_t stream) {
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int OTHER = F32 ? 12 : 24;
  const Form f = form_of(a.experts, F32);
  if (f.per == 8) return launch_k<T, 1, 8>(a, blocks, stream);
  if (f.per == 16) switch (f.threads) {
      case 1: return launch_k<T, 1, 16>(a, blocks, stream);
      case 2: return launch_k<T, 2, 16>(a, blocks, stream);
      case 4: return launch_k<T, 4, 16>(a, blocks, stream);
      case 8: return launch_k<T, 8, 16>(a, blocks, stream);
      case 16: return launch_k<T, 16, 16>(a, blocks, stream);
      case 32: return launch_k<T, 32, 16>(a, blocks, stream);
      default: return launch_k<T, 64, 16>(a, blocks, stream);
    }
  switch (f.threads) {
    case 1: return launch_k<T, 1, OTHER>(a, blocks, stream);
    case 2: return launch_k<T, 2, OTHER>(a, blocks, stream);
    case 4: return launch_k<T, 4, OTHER>(a, blocks, stream);
    case 8: return launch_k<T, 8, OTHER>(a, blocks, stream);
    case 16: return launch_k<T, 16, OTHER>(a, blocks, stream);
    case 32: return launch_k<T, 32, OTHER>(a, blocks, stream);
    default:
      if constexpr (F32) return launch_k<T, 64, OTHER>(a, blocks, stream);
  }
}

}  // namespace

// The launches of a type: route_f32.hip, route_bf16.hip, route_f16.hip
template <typename T>
void ds_route_rows(const void* args, unsigned blocks, hipStream_t stream);
template <typename T>
void ds_route_rows_backward(const void* args, unsigned blocks, hipStream_t stream);
