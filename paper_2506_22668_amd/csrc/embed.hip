// Rows of a table by id, and the table's gradient.
//
//   forward:   y[r] = s T[id_r],                          zeros where id_r is outside of [0, V)
//   backward:  dT[v] = s sum over r with id_r = v of dy[r],   zeros where there is none
//
// The gradient is summed by sorted ids: a stable radix sort of the pairs (id, r) on digits of up to 10 bits, then sums over stretches of equally many sorted
// rows, whatever ids they hold, so that an id with a large share of the rows costs as much as as many ids with one row. Where a stretch
// ends inside an id's rows it leaves a partial sum in fp32, and a last launch adds those up in order. Few rows are sorted and summed in one launch (few_sums_kernel).
// No atomic decides an order of floating-point sums: the same inputs give the same bits.
#include "feature_ops.h"
#include "group_range.h"
#include "rows.h"

namespace {

constexpr int kThreads = 256;

// ---- the rows -------------------------------------------------------------------------------------------------------------------------

struct LookArgs {
  int64_t rows;
  int cols, calls;      // pieces to a row
  int64_t rows_step;    // how far a thread's next piece is
  int calls_step, vocab;
  const int32_t* ids;
  const void* table;
  void* y;
  int64_t ts, ys;
  float scale;
};

constexpr int kAhead = 4;   // pieces of a thread on their way at a time: each waits for an id, and then for a row of the table

// A thread takes 16 bytes of y at a time and goes through the rows in steps of the whole launch; ids are asked for a round of kAhead pieces before they are needed. Bound by
// memory: 262,144 rows of 512 bf16 out of 100,003 of fp32 111 us, in which 537 MB of the table are read (a row comes up 2.6 times; some of it from the cache behind
// the L2s) and 268 MB written, 7.2 TB/s together; without ids ahead 113.
template <typename T, typename Y, bool TINY>
__global__ __launch_bounds__(kThreads) void look_up_kernel(LookArgs a) {
  constexpr int N = Piece<Y>::N;
  const int64_t first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int64_t row = first / a.calls;
  int call = (int)(first % a.calls);
  int64_t at[kAhead], next_at[kAhead];
  int col[kAhead], id[kAhead], next_col[kAhead], next_id[kAhead];
  const auto look = [&]() __attribute__((always_inline)) {   // the ids of the next pieces
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      next_at[j] = row;
      next_col[j] = call * N;
      next_id[j] = row < a.rows ? a.ids[row] : -1;
      row += a.rows_step;
      call += a.calls_step;
      if (call >= a.calls) {
        call -= a.calls;
        ++row;
      }
    }
  };
  look();
  while (next_at[0] < a.rows) {
    typename Elements<T, N>::V v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      at[j] = next_at[j];
      col[j] = next_col[j];
      id[j] = (uint32_t)next_id[j] < (uint32_t)a.vocab ? next_id[j] : -1;
      v[j] = load_elements<T, N, TINY>((const T*)a.table + (int64_t)(id[j] < 0 ? 0 : id[j]) * a.ts, col[j], a.cols);
    }
    look();
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (at[j] >= a.rows) break;
      settle_elements<T, N, TINY>(v[j], col[j], a.cols);
      PieceV<Y> out;
#pragma unroll
      for (int i = 0; i < N; ++i) out[i] = id[j] < 0 ? (Y)0.f : (Y)((float)v[j][i] * a.scale);
      store_piece<Y>((Y*)a.y + at[j] * a.ys + col[j], out, a.cols - col[j]);
    }
  }
}

template <typename T, typename Y>
void launch_look_up(ds_ctx* ctx, LookArgs& a) {
  constexpr int N = Piece<Y>::N;
  a.calls = (a.cols + N - 1) / N;
  const int64_t pieces = a.rows * a.calls, want = (pieces + kThreads - 1) / kThreads, most = 8 * (int64_t)ctx->num_cus;
  const int64_t blocks = want < most ? want : most, step = blocks * kThreads;
  a.rows_step = step / a.calls;
  a.calls_step = (int)(step % a.calls);
  const dim3 grid((unsigned)blocks), block(kThreads);
  if (a.cols < N) hipLaunchKernelGGL(HIP_KERNEL_NAME(look_up_kernel<T, Y, true>), grid, block, 0, ctx->stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(look_up_kernel<T, Y, false>), grid, block, 0, ctx->stream, a);
}

// ---- the sorted pairs -------------------------------------------------------------------------------------------------------------------
//
// A pass is three launches that wait for each other's counts, bound by latency: a million pairs into 50,021 ids in two passes of 8 bits 2 x (5.7 + 4.8 + 11.0 us); of the placing most is
// the scattered stores. Digits of up to 10 bits, since a thread has one and passes cost more than digits.

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMostBits = 10;      // of a digit: counts of 16 waves in 64 KB of LDS
constexpr int kStretch = 2048;     // rows of a workgroup, at the least, where there are several
constexpr int kMostBlocks = 256;
constexpr int kOwnBlocks = 32;     // up to which every workgroup adds up the others' counts itself; more have a launch for it (64,000 rows: 40.7 us so, 42.9 with it; 250,000: 64.4, 57.4)

struct SortArgs {
  const int32_t* ids;       // the first pass: the keys come from here, and rows are counted
  const int2* from;         // later ones: (key, row)
  int2* to;
  int rows, vocab, shift, bits, per_wave;
  int32_t* counts;          // [block][digits], and behind them the digits' rows where there are more than kOwnBlocks
  uint8_t* seen;            // [vocab], cleared by the first launch, set by the last pass where an id comes up
  bool mark;                // this is the last pass
};

__device__ __forceinline__ int2 pair_at(const SortArgs& a, int at) {
  if (!a.ids) return a.from[at];
  const int id = a.ids[at];
  return {(uint32_t)id < (uint32_t)a.vocab ? id : a.vocab, at};
}

// the pairs of one wave: a stretch of the rows
struct Stretch {
  int begin, end;
};
__device__ __forceinline__ Stretch stretch_of(const SortArgs& a, int block) {
  const int64_t first = ((int64_t)block * kSortWaves + (threadIdx.x >> 6)) * a.per_wave;
  Stretch s;
  s.begin = first < a.rows ? (int)first : a.rows;
  s.end = a.rows - s.begin < a.per_wave ? a.rows : s.begin + a.per_wave;
  return s;
}

constexpr int kHeld = 4;   // pairs of a thread that stay in its registers between counting and placing: all of them up to about a million rows

// counts of the workgroup's rows by wave and digit; the first kHeld pairs of a thread are left in `held`
__device__ __forceinline__ void count_digits(const SortArgs& a, const Stretch& s, int* count, int2 (&held)[kHeld]) {
  const int digits = 1 << a.bits, lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) held[j] = s.begin + j * 64 + lane < s.end ? pair_at(a, s.begin + j * 64 + lane) : int2{0, 0};
  for (int i = threadIdx.x; i < kSortWaves * digits; i += kSortThreads) count[i] = 0;
  __syncthreads();
  int* mine = count + (threadIdx.x >> 6) * digits;
  const auto add = [&](int key) { atomicAdd(&mine[key >> a.shift & (digits - 1)], 1); };   // (whole numbers: any order)
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (s.begin + j * 64 + lane < s.end) add(held[j].x);
  for (int at = s.begin + kHeld * 64 + lane; at < s.end; at += 64) add(pair_at(a, at).x);
  __syncthreads();
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs a, bool clear) {
  extern __shared__ int count[];
  if (clear)
    for (int64_t i = ((int64_t)blockIdx.x * kSortThreads + threadIdx.x) * 16; i < a.vocab; i += (int64_t)gridDim.x * kSortThreads * 16)
      *reinterpret_cast<uint4*>(a.seen + i) = uint4{0, 0, 0, 0};   // (its end is rounded up to 16 bytes)
  const int digits = 1 << a.bits;
  int2 held[kHeld];
  count_digits(a, stretch_of(a, (int)blockIdx.x), count, held);
  for (int d = threadIdx.x; d < digits; d += kSortThreads) {
    int n = 0;
    for (int w = 0; w < kSortWaves; ++w) n += count[w * digits + d];
    a.counts[(int)blockIdx.x * digits + d] = n;
  }
}

// Turns the workgroups' counts into the rows of the digit before each of them, and leaves the digits' rows behind them
__global__ __launch_bounds__(kSortThreads) void sort_before_kernel(SortArgs a, int blocks) {
  __shared__ int sum[kSortWaves][64];
  const int digits = 1 << a.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = (int)blockIdx.x * 64 + lane;
  const int each = (blocks + kSortWaves - 1) / kSortWaves, first = wave * each;
  int n[kMostBlocks / kSortWaves], all = 0;
#pragma unroll
  for (int j = 0; j < kMostBlocks / kSortWaves; ++j) n[j] = j < each && first + j < blocks && d < digits ? a.counts[(first + j) * digits + d] : 0;
#pragma unroll
  for (int j = 0; j < kMostBlocks / kSortWaves; ++j) all += n[j];
  sum[wave][lane] = all;
  __syncthreads();
  int before = 0, whole = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) {
    if (w < wave) before += sum[w][lane];
    whole += sum[w][lane];
  }
  if (d >= digits) return;
#pragma unroll
  for (int j = 0; j < kMostBlocks / kSortWaves; ++j) {
    if (j < each && first + j < blocks) a.counts[(first + j) * digits + d] = before;
    before += n[j];
  }
  if (wave == 0) a.counts[blocks * digits + d] = whole;
}

// One pass: each workgroup's pairs to their places. Lanes of one digit find each other by a ballot for each of its bits, so that a
// pair's rank is a popcount, and pairs of one digit keep their order.
__device__ __forceinline__ void place_pairs(const SortArgs& a, int block, int blocks, int* count, int* wave_sum) {
  const int digits = 1 << a.bits, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // (digits <= threads: thread d has digit d)
  const int d = (int)threadIdx.x;
  int whole = 0, before = 0;
  if (d < digits && blocks > kOwnBlocks) {
    before = a.counts[block * digits + d];
    whole = a.counts[blocks * digits + d];
  } else if (d < digits && blocks > 1) {
    for (int first = 0; first < blocks; first += 16) {
      int n[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) n[j] = first + j < blocks ? a.counts[(first + j) * digits + d] : 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        whole += n[j];
        before += first + j < block ? n[j] : 0;
      }
    }
  }
  const Stretch s = stretch_of(a, block);
  int2 held[kHeld];
  count_digits(a, s, count, held);
  if (d < digits && blocks == 1)
    for (int w = 0; w < kSortWaves; ++w) whole += count[w * digits + d];
  int upto = whole;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o, 64);
    if (lane >= o) upto += up;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  if (d < digits) {
    int at = upto - whole + before;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w)
      if (w < wave) at += wave_sum[w];
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = count[w * digits + d];
      count[w * digits + d] = at;
      at += c;
    }
  }
  __syncthreads();
  volatile int* mine = count + wave * digits;
  const auto place = [&](int2 now, bool there) __attribute__((always_inline)) {
    const int digit = now.x >> a.shift & (digits - 1);
    unsigned long long same = __ballot(there);
    for (int b = 0; b < a.bits; ++b) {
      const unsigned long long set = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    if (there) {
      const int rank = __popcll(same & ((1ull << lane) - 1)), at = mine[digit];
      a.to[at + rank] = now;
      if (a.mark && now.x < a.vocab) a.seen[now.x] = 1;
      if (rank == 0) mine[digit] = at + __popcll(same);   // (a wave's LDS accesses keep their order)
    }
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    if (s.begin + j * 64 >= s.end) return;
    place(held[j], s.begin + j * 64 + lane < s.end);
  }
  const int more = s.begin + kHeld * 64;
  int2 next = more + lane < s.end ? pair_at(a, more + lane) : int2{0, 0};
  for (int base = more; base < s.end; base += 64) {
    const int2 now = next;
    if (base + 64 + lane < s.end) next = pair_at(a, base + 64 + lane);
    place(now, base + lane < s.end);
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortArgs a) {
  extern __shared__ int count[];
  __shared__ int wave_sum[kSortWaves];
  place_pairs(a, (int)blockIdx.x, (int)gridDim.x, count, wave_sum);
}

__global__ __launch_bounds__(kThreads) void clear_kernel(uint8_t* seen, int vocab) {
  for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 16; i < vocab; i += (int64_t)gridDim.x * kThreads * 16)
    *reinterpret_cast<uint4*>(seen + i) = uint4{0, 0, 0, 0};   // (its end is rounded up to 16 bytes)
}

// ---- the sums -----------------------------------------------------------------------------------------------------------------------------

struct SumArgs {
  int rows, cols, vocab, share, chunk, chunks, calls;   // rows of a worker, and of a workgroup
  const int2* pairs;
  const int32_t* ids;   // few rows: not sorted yet
  int range;            //   and the ids of a workgroup
  const void* dy;
  void* dtable;
  int64_t dys, dts;
  float scale;
  uint8_t* seen;
  float* partial;       // [chunk][2][cols]: of the id that began before the chunk; of the one that goes on behind it
  int64_t rows_step;    // the pass over the table: how far a thread's next piece is
  int calls_step, clears;   // and its workgroups
};

constexpr int kRowsAhead = 8;

// N elements as the table has them, in pieces of 16 bytes
template <typename T, int N>
__device__ __forceinline__ void store_sums(T* to, const float (&v)[N], float scale, int have) {
  constexpr int P = Piece<T>::N;
#pragma unroll
  for (int p = 0; p < N / P; ++p) {
    PieceV<T> out;
#pragma unroll
    for (int i = 0; i < P; ++i) out[i] = (T)(v[p * P + i] * scale);
    store_piece<T>(to + p * P, out, have - p * P);
  }
}

// A thread's columns col .. of the sorted rows [begin, end): pair(i) is row i's (id, row), leave(id, sum, first, last) takes the sum of an id's rows, the first
// id's with `first` set, the last one's with `last`. Ids of `none` and beyond come last and are passed over.
template <typename D, bool TINY, typename Pair, typename Leave>
__device__ __forceinline__ void sum_rows(int begin, int end, int col, int cols, const D* dy, int64_t dys, int none, const Pair& pair, const Leave& leave) {
  constexpr int N = Piece<D>::N;
  float sum[N] = {};
  int2 now[kRowsAhead], next[kRowsAhead];
  typename Elements<D, N>::V v[kRowsAhead];
  int key = pair(begin).x;
  bool first = true;
#pragma unroll
  for (int j = 0; j < kRowsAhead; ++j) next[j] = pair(min(begin + j, end - 1));
  for (int at = begin; at < end; at += kRowsAhead) {
#pragma unroll
    for (int j = 0; j < kRowsAhead; ++j) {
      now[j] = next[j];
      v[j] = load_elements<D, N, TINY>(dy + now[j].y * dys, col, cols);
    }
    if (at + kRowsAhead < end) {
#pragma unroll
      for (int j = 0; j < kRowsAhead; ++j) next[j] = pair(min(at + kRowsAhead + j, end - 1));
    }
#pragma unroll
    for (int j = 0; j < kRowsAhead; ++j) {
      if (at + j >= end) break;
      if (now[j].x != key) {
        leave(key, sum, first, false);
        first = false;
        key = now[j].x;
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = 0.f;
      }
      if (key >= none) return;
      settle_elements<D, N, TINY>(v[j], col, cols);
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += (float)v[j][i];
    }
  }
  leave(key, sum, first, true);
}

// Clears the rows of ids that did not come up
template <typename T>
__device__ __forceinline__ void clear_rows(const SumArgs& a, int block) {
  constexpr int N = Piece<T>::N, AHEAD = 4;
  const int64_t first = (int64_t)block * kThreads + threadIdx.x;
  int64_t row = first / a.calls;
  int call = (int)(first % a.calls);
  while (row < a.vocab) {
    int64_t at[AHEAD];
    int col[AHEAD];
    bool empty[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      at[j] = row;
      col[j] = call * N;
      empty[j] = row < a.vocab && !a.seen[row];
      row += a.rows_step;
      call += a.calls_step;
      if (call >= a.calls) {
        call -= a.calls;
        ++row;
      }
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (empty[j]) store_piece<T>((T*)a.dtable + at[j] * a.dts + col[j], PieceV<T>{}, a.cols - col[j]);
  }
}

// LANES threads take a.share sorted rows, a piece of 16 bytes of their columns to a thread, and a workgroup a chunk: sums of ids that reach over a share's end meet in
// LDS, those of ids that reach over the chunk's go to memory. The first workgroups of the launch clear the rows of ids that did not come up beside it.
// Bound by memory: 1,000,175 rows of 128 bf16 into 50,021 of fp32 61 us, 4.7 TB/s.
template <typename D, typename T, int LANES, bool TINY>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumArgs a) {
  constexpr int N = Piece<D>::N, WORKERS = kThreads / LANES;
  __shared__ float meet[WORKERS][2][LANES * N];
  __shared__ bool through[WORKERS];   // one id has all of a worker's rows, and more on both sides
  if ((int)blockIdx.x < a.clears) {
    if (blockIdx.y == 0) clear_rows<T>(a, (int)blockIdx.x);
    return;
  }
  const int chunk = (int)blockIdx.x - a.clears, worker = (int)threadIdx.x / LANES, place = (int)threadIdx.x % LANES * N;
  const int col = (int)blockIdx.y * LANES * N + place, have = a.cols - col;
  const int64_t first_row = (int64_t)chunk * a.chunk + worker * a.share;
  const int begin = (int)min(first_row, (int64_t)a.rows), end = a.rows - begin < a.share ? a.rows : begin + a.share;
  T* dtable = (T*)a.dtable + col;
  bool before = false, after = false, whole = false;
  int key = 0;
  if (begin < end) {
    const int first_key = a.pairs[begin].x;
    key = a.pairs[end - 1].x;
    before = begin > 0 && a.pairs[begin - 1].x == first_key && first_key < a.vocab;   // the first id began before the share
    after = end < a.rows && a.pairs[end].x == key && key < a.vocab;                   // the last one goes on behind it
    whole = before && after && first_key == key;
    if (have > 0)
      sum_rows<D, TINY>(begin, end, col, a.cols, (const D*)a.dy, a.dys, a.vocab, [&](int i) { return a.pairs[i]; },
                        [&](int id, const float(&sum)[N], bool first, bool last) {
                          const bool goes_on = last && after, began = first && before;
                          if (goes_on || began) {
#pragma unroll
                            for (int i = 0; i < N; ++i) meet[worker][goes_on][place + i] = sum[i];
                          } else {
                            store_sums<T, N>(dtable + (int64_t)id * a.dts, sum, a.scale, have);
                          }
                        });
  }
  if (place == 0) through[worker] = whole;
  __syncthreads();
  if (have <= 0) return;
  float* partial = a.partial + (int64_t)chunk * 2 * a.cols + col;
  float sum[N];
  const auto take = [&](int w, int slot, bool more) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = more ? sum[i] + meet[w][slot][place + i] : meet[w][slot][place + i];
  };
  // the chunk's first id, where it began before and ends in the first share
  if (worker == 0 && before && !whole) {
    take(0, 0, false);
    store_sums<float, N>(partial, sum, 1.f, have);
  }
  // an id that goes on behind a share: its first worker here adds it up
  if (after && (worker == 0 || !whole)) {
    take(worker, 1, false);
    int w = worker + 1;
    while (w < WORKERS && through[w]) take(w++, 1, true);
    // (in the last share it goes on behind the chunk; else it ends in share w)
    if (w < WORKERS) {
      take(w, 0, true);
      if (whole) store_sums<float, N>(partial, sum, 1.f, have);
      else store_sums<T, N>(dtable + (int64_t)key * a.dts, sum, a.scale, have);
    } else {
      store_sums<float, N>(partial + a.cols, sum, 1.f, have);
    }
  }
}

// Adds up what the chunks left of ids that reach over a chunk's end, in order: a workgroup looks at kJoinChunks chunks and kJoinCols columns, kJoinLanes threads to an id that
// goes on over fewer than kShort chunks, all of them to a longer one. Bound by latency: 11.6 us behind the sums above, where most of the ids reach over one end alone.
constexpr int kJoinThreads = 512, kJoinChunks = 64, kJoinCols = 32, kJoinLanes = kJoinCols / 4, kJoinWorkers = kJoinThreads / kJoinLanes, kShort = 32;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void finish_kernel(SumArgs a, int col_tiles) {
  __shared__ int of_short[kJoinChunks], of_long[kJoinChunks], last_of[kJoinChunks], key_of[kJoinChunks], shorts, longs, last;
  __shared__ float meet[kJoinWorkers][kJoinCols];
  const int base = (int)blockIdx.x / col_tiles * kJoinChunks, col = (int)blockIdx.x % col_tiles * kJoinCols + (int)threadIdx.x % kJoinLanes * 4;
  const int worker = (int)threadIdx.x / kJoinLanes, have = a.cols - col;
  if (threadIdx.x == 0) shorts = longs = 0;
  if ((int)threadIdx.x < kJoinChunks) {
    // the id that begins in this chunk and goes on behind it; -1: none
    const int chunk = base + (int)threadIdx.x, begin = chunk < a.chunks ? chunk * a.chunk : a.rows;
    int found = -1;
    if (a.rows - begin > a.chunk) {
      const int end = begin + a.chunk, key = a.pairs[end - 1].x, behind = a.pairs[end].x, before = begin > 0 ? a.pairs[begin - 1].x : -1;
      if (key < a.vocab && behind == key && before != key) found = key;
    }
    key_of[threadIdx.x] = found;
  }
  __syncthreads();
  {
    // how far it goes, as far as kShort chunks: a wave looks at eight of the workgroup's chunks
    constexpr int EACH = kJoinChunks / (kJoinThreads / 64);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int start[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int chunk = base + wave * EACH + j + 1 + lane;
      start[j] = key_of[wave * EACH + j] >= 0 && chunk < a.chunks ? a.pairs[chunk * a.chunk].x : -2;
    }
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int c = wave * EACH + j;
      const unsigned long long other = __ballot(start[j] != key_of[c]);
      const int chunks = other ? __ffsll((long long)other) - 1 : 64;
      if (lane == 0 && key_of[c] >= 0) {
        last_of[c] = base + c + chunks;
        if (chunks < kShort) of_short[atomicAdd(&shorts, 1)] = c;   // (in any order: each has a result of its own)
        else of_long[atomicAdd(&longs, 1)] = c;
      }
    }
  }
  __syncthreads();
  // the sums of chunks from, from + step, .. upto, eight on their way at a time; a row's last columns are read where four end, and moved to their place
  const int at = have >= 4 ? col : max(a.cols - 4, 0), by = col - at;
  const auto add = [&](float (&sum)[4], int from, int upto, int step) __attribute__((always_inline)) {
    for (int c = from; c <= upto; c += 8 * step) {
      Elements<float, 4>::V v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int chunk = min(c + j * step, upto);
        const float* p = a.partial + ((int64_t)chunk * 2 + (chunk < upto)) * a.cols + at;
        if (a.cols >= 4) {
          v[j] = *reinterpret_cast<const Elements<float, 4>::U*>(p);
        } else {
#pragma unroll
          for (int i = 0; i < 3; ++i) v[j][i] = i < a.cols ? p[i] : 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j * step <= upto) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] += v[j][i];
        }
    }
    if (have > 0 && have < 4 && a.cols >= 4) {
#pragma unroll
      for (int s = 1; s < 4; ++s)
        if (by >= s) {
#pragma unroll
          for (int i = 0; i < 3; ++i) sum[i] = sum[i + 1];
        }
    }
  };
  const auto leave = [&](const float (&sum)[4], int key) __attribute__((always_inline)) {
    T* to = (T*)a.dtable + (int64_t)key * a.dts + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < have) to[i] = (T)(sum[i] * a.scale);
  };
  for (int s = worker; s < shorts; s += kJoinWorkers) {
    const int c = of_short[s];
    float sum[4] = {};
    add(sum, base + c, last_of[c], 1);
    leave(sum, key_of[c]);
  }
  for (int l = 0; l < longs; ++l) {
    const int chunk = base + of_long[l], key = key_of[of_long[l]];
    if (threadIdx.x == 0) last = 0;
    __syncthreads();
    int upto = last_of[of_long[l]];
    for (int c = upto + 1 + (int)threadIdx.x; c < a.chunks; c += 4 * kJoinThreads) {
      int start[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) start[j] = c + j * kJoinThreads < a.chunks ? a.pairs[(c + j * kJoinThreads) * a.chunk].x : -2;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (start[j] == key) upto = c + j * kJoinThreads;
      if (start[3] != key) break;
    }
    atomicMax(&last, upto);
    __syncthreads();
    upto = last;
    float sum[4] = {};
    add(sum, chunk + worker, upto, kJoinWorkers);
#pragma unroll
    for (int i = 0; i < 4; ++i) meet[worker][(int)threadIdx.x % kJoinLanes * 4 + i] = sum[i];
    __syncthreads();
    if (worker == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[i] = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWorkers; ++w) sum[i] += meet[w][(int)threadIdx.x * 4 + i];
      }
      leave(sum, key);
    }
    __syncthreads();
  }
}

// Few rows, in one launch: a workgroup has the ids [first, first + range) and the columns of its threads, finds its rows among all and sorts them in LDS, and its
// workers take equal shares of them. What ids that reach over a share's end leave meets in LDS. Every workgroup reads all ids, which is why rows are few: 1,010 rows of 64 fp32 into
// 2,000 5.3 us in one launch, 17.8 in the five of the other form (replayed from a graph); bound by latency.
constexpr int kFewThreads = 512, kFewWaves = kFewThreads / 64, kFewRange = 256;
constexpr int kFewRows = 8192;
static_assert(kFewRange <= 256 && kFewRows <= 1 << 24, "a pair is 32 bits");
template <typename D, typename T, int LANES, bool TINY>
__global__ __launch_bounds__(kFewThreads) void few_sums_kernel(SumArgs a) {
  constexpr int N = Piece<D>::N, WORKERS = kFewThreads / LANES, P = Piece<T>::N;
  __shared__ int count[kFewWaves][kFewRange], start[kFewRange + 1], wave_sum[kFewWaves];
  __shared__ uint32_t held[kFewRows];   // (digit, row)
  __shared__ float meet[WORKERS][2][LANES * N];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first_id = (int)blockIdx.x * a.range, range = min(a.range, a.vocab - first_id);
  for (int i = threadIdx.x; i < kFewWaves * kFewRange; i += kFewThreads) (&count[0][0])[i] = 0;
  __syncthreads();
  const int each = ((a.rows + kFewWaves - 1) / kFewWaves + 63) / 64 * 64, begin = min(wave * each, a.rows), end = min(begin + each, a.rows);
  const auto digit_of = [&](int row) { return row < end ? (uint32_t)a.ids[row] - (uint32_t)first_id : ~0u; };
  for (int row = begin + lane; row < end; row += 64) {
    const uint32_t digit = digit_of(row);
    if (digit < (uint32_t)range) atomicAdd(&count[wave][digit], 1);   // (whole numbers: any order)
  }
  __syncthreads();
  int own = 0, upto;
  if ((int)threadIdx.x < kFewRange)
    for (int w = 0; w < kFewWaves; ++w) own += count[w][threadIdx.x];
  upto = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o, 64);
    if (lane >= o) upto += up;
  }
  if (lane == 63) wave_sum[wave] = upto;
  __syncthreads();
  if ((int)threadIdx.x < kFewRange) {
    int at = upto - own;
    for (int w = 0; w < wave; ++w) at += wave_sum[w];
    start[threadIdx.x] = at;
    if (threadIdx.x == kFewRange - 1) start[kFewRange] = at + own;
    for (int w = 0; w < kFewWaves; ++w) {
      const int c = count[w][threadIdx.x];
      count[w][threadIdx.x] = at;
      at += c;
    }
  }
  __syncthreads();
  const int all = start[kFewRange];
  if (all > 0) {
    volatile int* mine = count[wave];
    for (int base = begin; base < end; base += 64) {
      const uint32_t digit = digit_of(base + lane);
      const bool there = digit < (uint32_t)range;
      unsigned long long same = __ballot(there);
      if (same == 0) continue;
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const unsigned long long set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
      }
      if (there) {
        const int rank = __popcll(same & ((1ull << lane) - 1)), at = mine[digit];
        held[at + rank] = digit << 24 | (uint32_t)(base + lane);
        if (rank == 0) mine[digit] = at + __popcll(same);   // (a wave's LDS accesses keep their order)
      }
    }
  }
  __syncthreads();
  T* dtable = (T*)a.dtable + (int64_t)first_id * a.dts;
  const int worker = (int)threadIdx.x / LANES, place = (int)threadIdx.x % LANES * N, col = (int)blockIdx.y * LANES * N + place, have = a.cols - col;
  const int share = (all + WORKERS - 1) / WORKERS, from = min(worker * share, all), to = min(from + share, all);
  const auto id_of = [&](int i) { return (int)(held[i] >> 24); };
  const bool before = from > 0 && from < to && id_of(from - 1) == id_of(from), after = to < all && from < to && id_of(to) == id_of(to - 1);
  if (have > 0) {
    for (int v = worker; v < range; v += WORKERS)
      if (start[v] == start[v + 1])
#pragma unroll
        for (int p = 0; p < N / P; ++p) store_piece<T>(dtable + (int64_t)v * a.dts + col + p * P, PieceV<T>{}, have - p * P);
    if (from < to)
      sum_rows<D, TINY>(from, to, col, a.cols, (const D*)a.dy, a.dys, a.range, [&](int i) { return int2{id_of(i), (int)(held[i] & 0xffffffu)}; },
                        [&](int key, const float(&sum)[N], bool first, bool last) {
                          const bool goes_on = last && after, began = first && before;
                          if (goes_on || began) {
#pragma unroll
                            for (int i = 0; i < N; ++i) meet[worker][goes_on][place + i] = sum[i];
                          } else {
                            store_sums<T, N>(dtable + (int64_t)key * a.dts + col, sum, a.scale, have);
                          }
                        });
  }
  __syncthreads();
  // an id that begins in this share and goes on behind it
  if (have > 0 && after && !(before && id_of(from) == id_of(to - 1))) {
    const int key = id_of(to - 1);
    float sum[N] = {};
    int w = worker;
    do {
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += meet[w][1][place + i];
      ++w;
    } while ((w + 1) * share < all && id_of((w + 1) * share) == key);
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] += meet[w][0][place + i];
    store_sums<T, N>(dtable + (int64_t)key * a.dts + col, sum, a.scale, have);
  }
}

// rows of a worker: enough workers for the card
int share_of(int rows) {
  int c = 16;
  while (c < 256 && (rows + c - 1) / c > 16384) c *= 2;
  return c;
}
int digits_of(int vocab, int* passes) {
  const int bits = 32 - __builtin_clz((unsigned)vocab);   // of 0 .. vocab
  *passes = (bits + kMostBits - 1) / kMostBits;
  return (bits + *passes - 1) / *passes;
}
int sort_blocks(int rows) {
  const int blocks = (rows + kStretch - 1) / kStretch;
  return blocks <= 2 ? 1 : blocks < kMostBlocks ? blocks : kMostBlocks;
}

// Few rows: ids of a workgroup, so that there are about 512 workgroups (of 64 columns or more); 0: another form. A workgroup takes all rows of its ids, in about 5 us and 8 more for
// each 1,000 of them, and the other form 17 to 30 us, more with more ids; how ids are spread is known on the GPU alone. In us, this form and the other, 128 columns of bf16:
//   rows   into 4,096 ids   1,024    128      32       8        1        4,096 ids, all rows of one
//   1,000  6 / 22           6 / 22   7 / 17   8 / 16   13 / 17  16 / 18  16 / 23
//   2,000  7 / 23           8 / 24   8 / 18   11 / 18  21 / 19  24 / 20  24 / 26
//   4,000  9 / 28           10 / 27  12 / 20  17 / 20  36 / 21  40 / 23  41 / 34
//   8,000  13 / 29          14 / 28  19 / 21  29 / 21  67 / 21  74 / 25  74 / 36
// (So many rows of few ids, evenly spread, to a workgroup at the most; and of fewer than 512 ids half as many in all, since more of them are likely to be of one.)
constexpr int kFewShare = 1024;
int few_range(int rows, int cols, int vocab) {
  if (rows > (vocab < 512 ? kFewRows / 2 : kFewRows)) return 0;
  const int64_t even = ((int64_t)vocab * ((cols + 63) / 64) + 511) / 512, range = even < 8 ? 8 : even;
  return range > kFewRange || (int64_t)rows * (range < vocab ? range : vocab) > (int64_t)kFewShare * vocab ? 0 : (int)range;
}

struct Layout {
  int64_t pairs, other, counts, seen, partial, bytes;
};
Layout layout_of(int rows, int cols, int vocab) {
  int passes;
  const int bits = digits_of(vocab, &passes), blocks = sort_blocks(rows);
  const int64_t least = 4 * share_of(rows), chunks = (rows + least - 1) / least;   // (four workers to a workgroup at the least)
  Layout l = {};
  if (few_range(rows, cols, vocab)) return l;
  int64_t at = 0;
  const auto place = [&](int64_t bytes) {
    const int64_t here = at;
    at += (bytes + 15) / 16 * 16;
    return here;
  };
  l.pairs = place((int64_t)rows * 8);
  l.other = place(passes > 1 ? (int64_t)rows * 8 : 0);
  l.counts = place(blocks > 1 ? (int64_t)(blocks + 1) * (1 << bits) * 4 : 0);
  l.seen = place(vocab);
  l.partial = place(chunks * 2 * cols * 4);
  l.bytes = at;
  return l;
}

int sort_ids(ds_ctx* ctx, const int32_t* ids, int rows, int vocab, int2* pairs, int2* other, int32_t* counts, uint8_t* seen) {
  int passes;
  SortArgs a = {};
  a.ids = ids;
  a.rows = rows;
  a.vocab = vocab;
  a.bits = digits_of(vocab, &passes);
  a.counts = counts;
  a.seen = seen;
  const int blocks = sort_blocks(rows), lds = kSortWaves * (1 << a.bits) * (int)sizeof(int);
  const int64_t waves = (int64_t)blocks * kSortWaves, each = (rows + waves - 1) / waves;
  a.per_wave = (int)((each + 63) / 64 * 64);
  if (lds > 48 * 1024) {
    DS_HIP(ctx, hipFuncSetAttribute((const void*)sort_count_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    DS_HIP(ctx, hipFuncSetAttribute((const void*)sort_place_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  }
  for (int p = 0; p < passes; ++p) {
    a.to = (passes - 1 - p) & 1 ? other : pairs;
    a.mark = p == passes - 1;
    if (blocks > 1) {
      hipLaunchKernelGGL(sort_count_kernel, dim3(blocks), dim3(kSortThreads), lds, ctx->stream, a, p == 0);
      if (blocks > kOwnBlocks)
        hipLaunchKernelGGL(sort_before_kernel, dim3(((1 << a.bits) + 63) / 64), dim3(kSortThreads), 0, ctx->stream, a, blocks);
    } else if (p == 0) {
      const int64_t clear = ((int64_t)vocab + 16 * kThreads - 1) / (16 * kThreads), most = 8 * (int64_t)ctx->num_cus;
      hipLaunchKernelGGL(clear_kernel, dim3((unsigned)(clear < most ? clear : most)), dim3(kThreads), 0, ctx->stream, seen, vocab);
    }
    hipLaunchKernelGGL(sort_place_kernel, dim3(blocks), dim3(kSortThreads), lds, ctx->stream, a);
    a.ids = nullptr;
    a.from = a.to;
    a.shift += a.bits;
  }
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

template <typename D, typename T, int LANES>
void launch_sum(SumArgs& a, hipStream_t stream) {
  constexpr int N = Piece<D>::N;
  a.chunk = a.share * (kThreads / LANES);
  a.chunks = (a.rows + a.chunk - 1) / a.chunk;
  const dim3 grid(a.clears + a.chunks, (a.cols + LANES * N - 1) / (LANES * N)), block(kThreads);
  if (a.cols < N) hipLaunchKernelGGL(HIP_KERNEL_NAME(sum_kernel<D, T, LANES, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(sum_kernel<D, T, LANES, false>), grid, block, 0, stream, a);
}

template <typename D, typename T>
int launch_sums(ds_ctx* ctx, SumArgs& a) {
  a.calls = (a.cols + Piece<T>::N - 1) / Piece<T>::N;
  const int64_t all = (int64_t)a.vocab * a.calls, want = (all + kThreads - 1) / kThreads, most = 4 * (int64_t)ctx->num_cus;
  a.clears = (int)(want < most ? want : most);
  const int64_t step = (int64_t)a.clears * kThreads;
  a.rows_step = step / a.calls;
  a.calls_step = (int)(step % a.calls);
  const int pieces = (a.cols + Piece<D>::N - 1) / Piece<D>::N, col_tiles = (a.cols + kJoinCols - 1) / kJoinCols;
  if (pieces <= 8) launch_sum<D, T, 8>(a, ctx->stream);
  else if (pieces <= 16) launch_sum<D, T, 16>(a, ctx->stream);
  else if (pieces <= 32) launch_sum<D, T, 32>(a, ctx->stream);
  else launch_sum<D, T, 64>(a, ctx->stream);
  const int64_t joins = (int64_t)((a.chunks + kJoinChunks - 1) / kJoinChunks) * col_tiles;
  if (joins > ds_most_workgroups(kJoinThreads)) return ds_fail(ctx, DS_EINVAL, "%d rows of %d columns are more than a launch has", a.rows, a.cols);
  if (a.chunks > 1) hipLaunchKernelGGL(HIP_KERNEL_NAME(finish_kernel<T>), dim3((unsigned)joins), dim3(kJoinThreads), 0, ctx->stream, a, col_tiles);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

template <typename D, typename T, int LANES>
void launch_few(const SumArgs& a, hipStream_t stream) {
  const dim3 grid((a.vocab + a.range - 1) / a.range, (a.cols + LANES * Piece<D>::N - 1) / (LANES * Piece<D>::N)), block(kFewThreads);
  if (a.cols < Piece<D>::N) hipLaunchKernelGGL(HIP_KERNEL_NAME(few_sums_kernel<D, T, LANES, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(few_sums_kernel<D, T, LANES, false>), grid, block, 0, stream, a);
}

template <typename D, typename T>
int launch_backward(ds_ctx* ctx, SumArgs& a) {
  if (a.range == 0) return launch_sums<D, T>(ctx, a);
  if (a.cols <= 8 * Piece<D>::N) launch_few<D, T, 8>(a, ctx->stream);
  else launch_few<D, T, 16>(a, ctx->stream);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

}  // namespace

int ds_launch_embed(ds_ctx* ctx, int dtype, int table_dtype, int64_t rows, int cols, int vocab, ds_rows table, const int32_t* ids, float scale, ds_rows y) {
  if (rows == 0) return DS_OK;
  LookArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.vocab = vocab;
  a.ids = ids;
  a.table = table.data;
  a.ts = table.stride;
  a.y = (void*)y.data;
  a.ys = y.stride;
  a.scale = scale;
  if (dtype == DS_ELEM_F32) launch_look_up<float, float>(ctx, a);
  else if (dtype == DS_ELEM_BF16) table_dtype == DS_ELEM_F32 ? launch_look_up<float, __bf16>(ctx, a) : launch_look_up<__bf16, __bf16>(ctx, a);
  else table_dtype == DS_ELEM_F32 ? launch_look_up<float, _Float16>(ctx, a) : launch_look_up<_Float16, _Float16>(ctx, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

int64_t ds_embed_backward_bytes(int rows, int cols, int vocab) { return layout_of(rows, cols, vocab).bytes; }

int ds_launch_embed_backward(ds_ctx* ctx, int dtype, int table_dtype, int rows, int cols, int vocab, ds_rows dy, const int32_t* ids, float scale,
                             ds_rows dtable, void* workspace) {
  const Layout l = layout_of(rows, cols, vocab);
  char* base = (char*)workspace;
  int2* pairs = (int2*)(base + l.pairs);
  uint8_t* seen = (uint8_t*)(base + l.seen);
  SumArgs a = {};
  a.rows = rows;
  a.cols = cols;
  a.vocab = vocab;
  a.share = share_of(rows);
  a.pairs = pairs;
  a.dy = dy.data;
  a.dys = dy.stride;
  a.dtable = (void*)dtable.data;
  a.dts = dtable.stride;
  a.scale = scale;
  a.seen = seen;
  a.partial = (float*)(base + l.partial);
  a.ids = ids;
  a.range = few_range(rows, cols, vocab);
  if (a.range == 0) DS_TRY(sort_ids(ctx, ids, rows, vocab, pairs, (int2*)(base + l.other), (int32_t*)(base + l.counts), seen));
  if (dtype == DS_ELEM_F32) return launch_backward<float, float>(ctx, a);
  if (dtype == DS_ELEM_BF16) return table_dtype == DS_ELEM_F32 ? launch_backward<__bf16, float>(ctx, a) : launch_backward<__bf16, __bf16>(ctx, a);
  return table_dtype == DS_ELEM_F32 ? launch_backward<_Float16, float>(ctx, a) : launch_backward<_Float16, _Float16>(ctx, a);
}
