// Products of rows with the weights of their group where a group has many rows: tiles through LDS.
#include "grouped_mm.h"
#include "mm_split.h"
#include "rows.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define DS_LDS __attribute__((address_space(3)))
#define DS_GLOBAL __attribute__((address_space(1)))

constexpr int kDepthBytes = 128;   // of a step of the contraction

__device__ const uint4 kZeros = {0, 0, 0, 0};

template <typename T>
using PieceV = typename Piece<T>::V;

__device__ __forceinline__ f32x16 multiply(PieceV<__bf16> a, PieceV<__bf16> b, f32x16 d) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(PieceV<_Float16> a, PieceV<_Float16> b, f32x16 d) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(PieceV<float> a, PieceV<float> b, f32x16 d) {
#pragma unroll
  for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], d, 0, 0, 0);
  return d;
}

// column of the tile that row m of a matrix-core operand stands for: a lane's 16 results are then 16 neighbours
__device__ __forceinline__ int column_of(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

// An operand in LDS. ACROSS false: [COLS][128 bytes of the contraction], 16-byte pieces of a column exchanged by its last three bits;
// true: [steps of the contraction][COLS], pieces exchanged by the step's last two bits (16-bit types).
template <typename T, int COLS, bool ACROSS>
struct Operand {
  static constexpr int N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T), BYTES = COLS * kDepthBytes;
  static constexpr int PER_ROW = ACROSS ? COLS / N : 8;
  // the place of piece number `at` of the tile: its column (or step) and which piece of that
  static __device__ __forceinline__ int line(int at) { return at / PER_ROW; }
  static __device__ __forceinline__ int piece(int at) {
    const int p = at % PER_ROW;
    if constexpr (ACROSS) return sizeof(T) == 2 ? p ^ ((line(at) & 3) << 2) : p;
    else return p ^ (line(at) & 7);
  }
};

// A lane's operand pieces for 32 columns and 2 N steps of the contraction
template <typename T, int COLS, bool ACROSS, bool ORDERED>
struct Reader {
  using Op = Operand<T, COLS, ACROSS>;
  int m, h, lane;
  __device__ __forceinline__ Reader(int lane_) : lane(lane_) {
    const int r = lane & 31;
    m = ORDERED ? column_of(r) : r;
    h = lane >> 5;
  }
  // columns first .. first + 31, steps slice * 2 N ..
  __device__ __forceinline__ PieceV<T> read(const char* tile, int first, int slice) const {
    constexpr int N = Op::N;
    if constexpr (!ACROSS) {
      return *reinterpret_cast<const PieceV<T>*>(tile + (first + m) * kDepthBytes + (((2 * slice + h) ^ (m & 7)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      const int i = lane & 15, four = ((lane >> 4) & 1) * 4 + (i & 3);
      const int col = first + (ORDERED ? 16 * (four & 1) + 4 * (four >> 1) : 4 * four);
      const int byte = (slice * 16 + 8 * h + (i >> 2)) * (COLS * 2) + (((col >> 3) ^ ((i >> 2) << 2)) << 4) + (col & 7) * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DS_LDS s16x4*)(tile + byte));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DS_LDS s16x4*)(tile + byte + 4 * COLS * 2));
      union {
        s16x4 half[2];
        PieceV<T> whole;
      } u;
      u.half[0] = lo;
      u.half[1] = hi;
      return u.whole;
    } else {
      PieceV<T> v;
#pragma unroll
      for (int i = 0; i < N; ++i)
        v[i] = *reinterpret_cast<const float*>(tile + (slice * 2 * N + N * h + i) * (COLS * 4) + (first + m) * 4);
      return v;
    }
  }
};

// Brings pieces of an operand into LDS: piece u of thread t is piece number u * THREADS + t of the tile. Direct loads go there by
// themselves; rows that are not aligned for them come through registers.
template <typename T, int COLS, int THREADS, bool DIRECT>
struct Loader {
  static constexpr int N = Piece<T>::N, PIECES = COLS * kDepthBytes / 16 / THREADS;
  PieceV<T> held[DIRECT ? 1 : PIECES];

  // have: elements that there are from p on (zeros behind them)
  __device__ __forceinline__ void fetch(int u, const T* p, int have, char* tile) {
    if constexpr (DIRECT) {
      const T* src = have > 0 ? p : reinterpret_cast<const T*>(&kZeros);
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      __builtin_amdgcn_global_load_lds((const DS_GLOBAL void*)src, (DS_LDS void*)(tile + (u * THREADS + wave * 64) * 16), 16, 0, 0);
    } else {
      held[u] = load_piece<T>(p, have);
    }
  }
  __device__ __forceinline__ void store(char* tile) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int u = 0; u < PIECES; ++u) *reinterpret_cast<PieceV<T>*>(tile + (u * THREADS + (int)threadIdx.x) * 16) = held[u];
    }
  }
};

// Workgroups stay: one to a compute unit, which goes through tiles of BR rows and BN columns. A step of the contraction (128 bytes of
// every row) is computed on from one half of the LDS while the next but one comes into the other; a wave's operands for a slice of the
// step are read while the matrix cores work on the slice before.
template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WN, 2) void row_tiles_kernel(MmArgs a) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T);
  constexpr int TR = BR / WR, TN = BN / WN, NR = TR / 32, NN = TN / 32, SLICES = DEPTH / (2 * N);
  constexpr int SHIFT = BR == 256 ? 8 : BR == 128 ? 7 : 6;
  using XOp = Operand<T, BR, false>;
  using WOp = Operand<T, BN, !TRANSPOSED>;
  constexpr int STAGE = XOp::BYTES + WOp::BYTES;
  // results on their way out: a wave's rows, PASS blocks of 32 at a time, lie in `odd`
  constexpr int OUT_ROW = TN * (int)sizeof(T), PASS = STAGE / (WR * WN) / (32 * OUT_ROW) < NR ? STAGE / (WR * WN) / (32 * OUT_ROW) : NR;
  constexpr int CHUNKS = OUT_ROW / 16, ROWS_AT_ONCE = 64 / CHUNKS;
  // (two arrays, not halves of one: only then does the compiler know that what is read of one does not wait for what comes into the other)
  __shared__ __attribute__((aligned(128))) char even[STAGE], odd[STAGE];
  __shared__ int row_of[2][BR];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (wave / WN) * TR, wn = (wave % WN) * TN;
  const int width = TRANSPOSED ? a.inner : a.outer, depth = TRANSPOSED ? a.outer : a.inner;
  const T* x = (const T*)(TRANSPOSED ? a.dy : a.x);
  const int64_t xs = TRANSPOSED ? a.dys : a.xs;
  const T* gate = (const T*)a.gate;
  T* y = (T*)a.y;
  GroupTiles all(a.offsets, a.groups, a.rows, SHIFT);
  // Workgroups go to the eight XCDs in turn. Each XCD has a stretch of the tiles, column tiles of a row tile next to each other, so that they
  // share its L2; its workgroups take them in turn.
  const int64_t tiles = (int64_t)all.count() * a.col_tiles;
  const int xcd = (int)blockIdx.x & 7, step_by = (int)gridDim.x >> 3;
  const int64_t stretch = tiles * (xcd + 1) / 8;
  int64_t at = tiles * xcd / 8 + ((int)blockIdx.x >> 3);

  Loader<T, BR, THREADS, DIRECT> lx;
  Loader<T, BN, THREADS, DIRECT> lw;
  const Reader<T, BR, false, false> rx(lane);
  const Reader<T, BN, !TRANSPOSED, true> rw(lane);
  const int steps = (depth + DEPTH - 1) / DEPTH;
  // A thread's pieces of a step lie in one place of lines that are a fixed number apart (the exchange of pieces goes by the last bits
  // of a line, which that number leaves alone)
  constexpr int XLINES = THREADS / XOp::PER_ROW, WLINES = THREADS / WOp::PER_ROW;
  static_assert(XLINES % 8 == 0 && WLINES % 8 == 0, "");
  const int xk = XOp::piece((int)threadIdx.x) * N, wline = WOp::line((int)threadIdx.x), wplace = WOp::piece((int)threadIdx.x) * N;
  const T *from_x[lx.PIECES], *from_w;
  GroupTile gt;
  int col0, turn = 0;
  const auto fetch = [&](int s, char* stage) {
    const int k = s * DEPTH;
#pragma unroll
    for (int u = 0; u < lw.PIECES; ++u) {
      const int line = u * WLINES + wline;
      if constexpr (TRANSPOSED) lw.fetch(u, from_w + (int64_t)(u * WLINES) * a.outer + k, col0 + line < width ? depth - k - wplace : 0, stage);
      else lw.fetch(u, from_w + (int64_t)(k + u * WLINES) * a.outer, k + line < depth ? width - col0 - wplace : 0, stage);
    }
#pragma unroll
    for (int u = 0; u < lx.PIECES; ++u) lx.fetch(u, from_x[u] + k, depth - k - xk, stage + WOp::BYTES);
  };
  const auto put = [&](char* stage) {
    lw.store(stage);
    lx.store(stage + WOp::BYTES);
  };
  // what a thread brings of tile `at`, and its first step
  const auto start = [&]() {
    gt = all.find((int)(at / a.col_tiles));
    col0 = (int)(at % a.col_tiles) * BN;
    turn ^= 1;
    if (threadIdx.x < BR) {
      const int pos = gt.begin + (int)threadIdx.x;
      row_of[turn][threadIdx.x] = pos < gt.end ? ds_ordered_row(a.order, a.rows, pos) : -1;
    }
    if (gt.group == a.groups) return;
#pragma unroll
    for (int u = 0; u < lx.PIECES; ++u) {
      const int pos = gt.begin + u * XLINES + XOp::line((int)threadIdx.x);
      const int r = pos < gt.end ? ds_ordered_row(a.order, a.rows, pos) : 0;
      from_x[u] = x + (r < 0 ? 0 : r) * xs + xk;   // (no row: any row, whose results go nowhere)
    }
    from_w = (const T*)a.w + (int64_t)gt.group * a.inner * a.outer +
             (TRANSPOSED ? (int64_t)(col0 + wline) * a.outer + wplace : (int64_t)wline * a.outer + col0 + wplace);
    fetch(0, even);
    put(even);
  };

  if (at >= stretch) return;
  start();
  while (true) {
    f32x16 acc[NR][NN] = {};
    if (gt.group < a.groups) {
      PieceV<T> fx[2][NR], fw[2][NN];
      const auto read = [&](const char* stage, int c) {
#pragma unroll
        for (int n = 0; n < NN; ++n) fw[c & 1][n] = rw.read(stage, wn + n * 32, c);
#pragma unroll
        for (int r = 0; r < NR; ++r) fx[c & 1][r] = rx.read(stage + WOp::BYTES, wr + r * 32, c);
      };
      const auto work = [&](int c) {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int n = 0; n < NN; ++n) acc[r][n] = multiply(fw[c & 1][n], fx[c & 1][r], acc[r][n]);
      };
      const auto step = [&](int s, char* now, char* then) {
#pragma unroll
        for (int c = 0; c + 1 < SLICES; ++c) {
          read(now, c + 1);
          __builtin_amdgcn_sched_barrier(0);
          work(c);
          __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();   // step s + 1 is there, and nobody reads step s any more
        if (s + 2 < steps) {
          put(now);
          fetch(DIRECT ? s + 2 : s + 3, now);
        }
        if (s + 1 < steps) {
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int n = 0; n < NN; ++n) fw[0][n] = rw.read(then, wn + n * 32, 0);
#pragma unroll
          for (int r = 0; r < NR; ++r) fx[0][r] = rx.read(then + WOp::BYTES, wr + r * 32, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
        work(SLICES - 1);
      };
      static_assert(SLICES % 2 == 0, "");
      if (steps > 1) {
        fetch(1, odd);
        put(odd);
        if (!DIRECT) fetch(2, even);
      }
      __syncthreads();
      read(even, 0);
      for (int s = 0; s < steps; s += 2) {
        step(s, even, odd);
        if (s + 1 < steps) step(s + 1, odd, even);
      }
    }
    // the next tile's first step comes in while this one's results go out
    const GroupTile done = gt;
    const int col = col0 + wn, ids = turn;
    at += step_by;
    const bool more = at < stretch;
    __syncthreads();
    if (more) start();
    char* mine = odd + wave * (STAGE / (WR * WN));
#pragma unroll
    for (int r0 = 0; r0 < NR; r0 += PASS) {
#pragma unroll
      for (int n = 0; n < NN; ++n) {
        const int c = col + n * 32 + 16 * (lane >> 5);
        float bias[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          bias[i] = a.bias && done.group < a.groups && c + i < width ? a.bias[(int64_t)done.group * width + c + i] : 0.f;
#pragma unroll
        for (int r = 0; r < PASS; ++r)
#pragma unroll
          for (int p = 0; p < 16 / N; ++p) {
            PieceV<T> out;
#pragma unroll
            for (int i = 0; i < N; ++i) {
              float v = acc[r0 + r][n][p * N + i] + bias[p * N + i];
              if (a.relu) v = v < 0.f ? 0.f : v;   // (a NaN stays one)
              out[i] = (T)v;
            }
            const int line = r * 32 + (lane & 31), chunk = (n * 32 + 16 * (lane >> 5)) / N + p;
            *reinterpret_cast<PieceV<T>*>(mine + line * OUT_ROW + ((chunk ^ (line & 7)) << 4)) = out;
          }
      }
      // (a wave reads what it wrote itself: its LDS accesses keep their order)
#pragma unroll
      for (int i = 0; i < PASS * 32 / ROWS_AT_ONCE; ++i) {
        const int line = i * ROWS_AT_ONCE + lane / CHUNKS, chunk = lane % CHUNKS, c = col + chunk * N;
        const int row = row_of[ids][wr + r0 * 32 + line];
        PieceV<T> out = *reinterpret_cast<const PieceV<T>*>(mine + line * OUT_ROW + ((chunk ^ (line & 7)) << 4));
        if (row >= 0 && c < width) {
          if (gate) {
            const PieceV<T> open = load_piece<T>(gate + row * a.gs + c, width - c);
#pragma unroll
            for (int j = 0; j < N; ++j) out[j] = (float)open[j] > 0.f ? out[j] : (T)0.f;
          }
          store_piece<T>(y + row * a.ys + c, out, width - c);
        }
      }
    }
    if (!more) return;
    __syncthreads();
  }
}

template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED, bool DIRECT>
int launch_one(ds_ctx* ctx, MmArgs& a) {
  a.col_tiles = ((TRANSPOSED ? a.inner : a.outer) + BN - 1) / BN;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(row_tiles_kernel<T, BR, BN, WR, WN, TRANSPOSED, DIRECT>), dim3((unsigned)(ctx->num_cus + 7) / 8 * 8),
                     dim3(64 * WR * WN), 0, ctx->stream, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

bool sixteen(const void* p, int64_t stride, size_t element) { return (uintptr_t)p % 16 == 0 && stride * element % 16 == 0; }

// ---- the gradient of the weights ------------------------------------------------------------------------------------------------
// dW_g = sum_r x[r]^T dy[r]: both operands run across the contraction, which is the group's rows. Groups are ragged and there are about
// as many tiles as compute units, so the steps of all tiles of all groups lie in one line (group by group, tile by tile) that is cut
// evenly, a stretch to a workgroup. Where a cut falls inside a tile, the workgroups on both sides leave fp32 sums (at most two a
// workgroup), which a second launch adds up in order: no atomics, the same bits every time.
// the steps of a group's contraction
__device__ __forceinline__ int group_steps(const MmArgs& a, int g, int depth, int* begin, int* end) {
  ds_group_range(a.offsets, a.groups, a.rows, g, begin, end);
  return (*end - *begin + depth - 1) / depth;
}

// Steps of all groups (each tile's), and where unit `unit` of the line falls: its group (-1: behind the end) and the steps before it
// there, of all tiles. Called by whole waves, the same answer in every lane.
__device__ __forceinline__ int64_t locate_unit(const MmArgs& a, int depth, int tiles, int64_t unit, int* group, int64_t* within) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  *group = -1;
  for (int base = 0; base < a.groups; base += 64) {
    int begin, end;
    const int g = base + lane;
    const int64_t own = g < a.groups ? (int64_t)group_steps(a, g, depth, &begin, &end) * tiles : 0;
    int64_t upto = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t up = __shfl_up(upto, o, 64);
      if (lane >= o) upto += up;
    }
    const unsigned long long reach = __ballot(before + upto > unit);
    if (reach && *group < 0) {
      const int src = __ffsll((long long)reach) - 1;
      *group = __builtin_amdgcn_readfirstlane(base + src);
      *within = unit - __shfl(before + upto - own, src, 64);
    }
    before += __shfl(upto, 63, 64);
  }
  return before;
}

template <typename T, int BR, int BN, int WR, int WN, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WN, 2) void weight_tiles_kernel(MmArgs a, float* partial) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T);
  constexpr int NR = BR / WR / 32, NN = BN / WN / 32, SLICES = DEPTH / (2 * N), SLOT = BR * BN + BN;
  using XOp = Operand<T, BR, true>;
  using DOp = Operand<T, BN, true>;
  constexpr int STAGE = XOp::BYTES + DOp::BYTES;
  constexpr int PARTS = THREADS / BN, EACH = DEPTH / PARTS;   // of the sums for db: threads to a column, steps of each
  __shared__ __attribute__((aligned(128))) char even[STAGE], odd[STAGE];
  __shared__ float sums[PARTS][BN];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = (wave / WN) * (BR / WR), wn = (wave % WN) * (BN / WN);
  const int tiles = (a.inner + BR - 1) / BR * a.col_tiles;
  int group;
  int64_t within, dummy;
  int none;
  const int64_t units = locate_unit(a, DEPTH, tiles, 0, &none, &dummy);
  const int64_t wgs = units < (int64_t)gridDim.x ? units : (int64_t)gridDim.x;   // (none without a unit: the join reads all that there are)
  if ((int64_t)blockIdx.x >= wgs) return;
  int64_t unit = ds_mm_even_begin(blockIdx.x, wgs, units);
  const int64_t last = ds_mm_even_begin(blockIdx.x + 1, wgs, units);
  locate_unit(a, DEPTH, tiles, unit, &group, &within);
  const T *x = (const T*)a.x, *dy = (const T*)a.dy;
  const Reader<T, BR, true, false> rx(lane);
  const Reader<T, BN, true, true> rd(lane);
  while (unit < last && group < a.groups) {
    int begin, end;
    const int steps = group_steps(a, group, DEPTH, &begin, &end);
    if (within >= (int64_t)steps * tiles) {   // on to the next group
      ++group;
      within = 0;
      continue;
    }
    const int tile = (int)(within / steps), first = (int)(within % steps);
    const int upto = last - unit < steps - first ? first + (int)(last - unit) : steps;
    const int in0 = tile / a.col_tiles * BR, col0 = tile % a.col_tiles * BN;
    f32x16 acc[NR][NN] = {};
    float sum = 0.f;
    Loader<T, BR, THREADS, DIRECT> lx;
    Loader<T, BN, THREADS, DIRECT> ld;
    constexpr int LINES = THREADS / XOp::PER_ROW;   // (as in row_tiles_kernel)
    static_assert(BR == BN && LINES % 4 == 0, "both operands' pieces of a thread lie in the same rows");
    int row[lx.PIECES];
    const int line = XOp::line((int)threadIdx.x), place = XOp::piece((int)threadIdx.x) * N;
    const T *from_x = x + in0 + place, *from_dy = dy + col0 + place;
    const auto find_rows = [&](int s) {
#pragma unroll
      for (int u = 0; u < lx.PIECES; ++u) {
        const int pos = begin + s * DEPTH + u * LINES + line;
        row[u] = s < upto && pos < end ? ds_ordered_row(a.order, a.rows, pos) : -1;
      }
    };
    const auto fetch = [&](char* stage) {
#pragma unroll
      for (int u = 0; u < ld.PIECES; ++u) ld.fetch(u, from_dy + row[u] * a.dys, row[u] < 0 ? 0 : a.outer - col0 - place, stage);
#pragma unroll
      for (int u = 0; u < lx.PIECES; ++u) lx.fetch(u, from_x + row[u] * a.xs, row[u] < 0 ? 0 : a.inner - in0 - place, stage + DOp::BYTES);
    };
    const auto step = [&](int s, char* now, char* then) {
      __syncthreads();
      if (s + 1 < upto) {
        fetch(then);
        find_rows(s + 2);
      }
#pragma unroll
      for (int c = 0; c < SLICES; ++c) {
        PieceV<T> fx[NR], fd[NN];
#pragma unroll
        for (int r = 0; r < NR; ++r) fx[r] = rx.read(now + DOp::BYTES, wr + r * 32, c);
#pragma unroll
        for (int n = 0; n < NN; ++n) fd[n] = rd.read(now, wn + n * 32, c);
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int n = 0; n < NN; ++n) acc[r][n] = multiply(fd[n], fx[r], acc[r][n]);
      }
      if (in0 == 0) {   // db: the column sums of what is in LDS anyway
        const int col = (int)threadIdx.x % BN, part = (int)threadIdx.x / BN;
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
          const int at = part * EACH + k;
          const int p = sizeof(T) == 2 ? (col / N) ^ ((at & 3) << 2) : col / N;
          v += (float)*reinterpret_cast<const T*>(now + at * (BN * (int)sizeof(T)) + p * 16 + col % N * (int)sizeof(T));
        }
        sum += v;
      }
      if (s + 1 < upto) {
        ld.store(then);
        lx.store(then + DOp::BYTES);
      }
    };
    __syncthreads();   // (the last tile's readers are through)
    find_rows(first);
    fetch(even);
    find_rows(first + 1);
    ld.store(even);
    lx.store(even + DOp::BYTES);
    for (int s = first; s < upto; s += 2) {
      step(s, even, odd);
      if (s + 1 < upto) step(s + 1, odd, even);
    }
    if (in0 == 0) {
      sums[threadIdx.x / BN][threadIdx.x % BN] = sum;
      __syncthreads();
      if (threadIdx.x < BN) {
        sum = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) sum += sums[p][threadIdx.x];
      }
    }
    if (first == 0 && upto == steps) {
      T* dw = (T*)a.dw + (int64_t)group * a.inner * a.outer;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const int in = in0 + wr + r * 32 + (lane & 31);
#pragma unroll
        for (int n = 0; n < NN; ++n)
#pragma unroll
          for (int p = 0; p < 16 / N; ++p) {
            const int c = col0 + wn + n * 32 + 16 * (lane >> 5) + p * N;
            if (in < a.inner && c < a.outer) {
              PieceV<T> out;
#pragma unroll
              for (int i = 0; i < N; ++i) out[i] = (T)acc[r][n][p * N + i];
              store_piece<T>(dw + (int64_t)in * a.outer + c, out, a.outer - c);
            }
          }
      }
      if (in0 == 0 && threadIdx.x < BN && col0 + (int)threadIdx.x < a.outer) a.db[(int64_t)group * a.outer + col0 + threadIdx.x] = sum;
    } else {
      // slot 0: the tile began with an earlier workgroup; 1: it begins here and a later one goes on
      float* to = partial + ((int64_t)blockIdx.x * 2 + (first == 0)) * SLOT;
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int n = 0; n < NN; ++n)
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const float4 v = {acc[r][n][4 * p], acc[r][n][4 * p + 1], acc[r][n][4 * p + 2], acc[r][n][4 * p + 3]};
            reinterpret_cast<float4*>(to)[((r * NN + n) * 4 + p) * THREADS + threadIdx.x] = v;
          }
      if (in0 == 0 && threadIdx.x < BN) to[BR * BN + threadIdx.x] = sum;
    }
    unit += upto - first;
    within += upto - first;
  }
}

// Adds up the sums of tiles that were cut, and clears the gradients of empty groups: a workgroup to a tile and 32 x 32 block of each wave
template <typename T, int BR, int BN, int WR, int WN>
__global__ __launch_bounds__(64 * WR * WN) void weight_join_kernel(MmArgs a, const float* partial, int wgs) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T);
  constexpr int NR = BR / WR / 32, NN = BN / WN / 32, SLOT = BR * BN + BN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = (wave / WN) * (BR / WR), wn = (wave % WN) * (BN / WN);
  const int tiles = (a.inner + BR - 1) / BR * a.col_tiles;
  const int group = (int)blockIdx.y, tile = (int)blockIdx.x / (NR * NN), block = (int)blockIdx.x % (NR * NN), r = block / NN, n = block % NN;
  const int in0 = tile / a.col_tiles * BR, col0 = tile % a.col_tiles * BN;
  int begin, end;
  const int steps = group_steps(a, group, DEPTH, &begin, &end);
  int64_t first = 0, last = -1, from = 0;
  if (steps > 0) {
    // where the tile's steps lie in the line: those of the groups before it first
    int64_t mine = 0, all = 0;
    for (int g = lane; g < a.groups; g += 64) {
      int b, e;
      const int64_t own = (int64_t)group_steps(a, g, DEPTH, &b, &e) * tiles;
      all += own;
      if (g < group) mine += own;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      all += __shfl_xor(all, o, 64);
      mine += __shfl_xor(mine, o, 64);
    }
    from = mine + (int64_t)tile * steps;
    const int64_t shares = all < wgs ? all : wgs;
    first = ds_mm_even_owner(from, shares, all);
    last = ds_mm_even_owner(from + steps - 1, shares, all);
    if (first == last) return;
  }
  f32x16 v = {};
  float sum = 0.f;
  const bool with_sum = in0 == 0 && block == 0 && threadIdx.x < BN;
  for (int64_t b = first; b <= last; ++b) {
    const float* p = partial + (b * 2 + (b == first)) * SLOT;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 f = reinterpret_cast<const float4*>(p)[(block * 4 + q) * THREADS + threadIdx.x];
      v[4 * q] += f.x;
      v[4 * q + 1] += f.y;
      v[4 * q + 2] += f.z;
      v[4 * q + 3] += f.w;
    }
    if (with_sum) sum += p[BR * BN + threadIdx.x];
  }
  T* dw = (T*)a.dw + (int64_t)group * a.inner * a.outer;
  const int in = in0 + wr + r * 32 + (lane & 31);
#pragma unroll
  for (int p = 0; p < 16 / N; ++p) {
    const int c = col0 + wn + n * 32 + 16 * (lane >> 5) + p * N;
    if (in < a.inner && c < a.outer) {
      PieceV<T> out;
#pragma unroll
      for (int i = 0; i < N; ++i) out[i] = (T)v[p * N + i];
      store_piece<T>(dw + (int64_t)in * a.outer + c, out, a.outer - c);
    }
  }
  if (with_sum && col0 + (int)threadIdx.x < a.outer) a.db[(int64_t)group * a.outer + col0 + threadIdx.x] = sum;
}

constexpr int kWeightGroups = 256;   // workgroups of the even cut

template <typename T, int BR, int BN, int WR, int WN>
int launch_weights(ds_ctx* ctx, MmArgs& a, float* partial) {
  a.col_tiles = (a.outer + BN - 1) / BN;
  const int64_t blocks = (int64_t)((a.inner + BR - 1) / BR) * a.col_tiles * (BR / WR / 32) * (BN / WN / 32);
  if (blocks > 0x7fffffff) return ds_fail(ctx, DS_EINVAL, "weights of %d by %d are more tiles than a launch has", a.inner, a.outer);
  const bool direct = sixteen(a.x, a.xs, sizeof(T)) && sixteen(a.dy, a.dys, sizeof(T)) && a.inner % Piece<T>::N == 0 && a.outer % Piece<T>::N == 0;
  const dim3 block(64 * WR * WN);
  if (direct) hipLaunchKernelGGL(HIP_KERNEL_NAME(weight_tiles_kernel<T, BR, BN, WR, WN, true>), dim3(kWeightGroups), block, 0, ctx->stream, a, partial);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(weight_tiles_kernel<T, BR, BN, WR, WN, false>), dim3(kWeightGroups), block, 0, ctx->stream, a, partial);
  hipLaunchKernelGGL(HIP_KERNEL_NAME(weight_join_kernel<T, BR, BN, WR, WN>), dim3((unsigned)blocks, a.groups), block, 0, ctx->stream, a, partial, kWeightGroups);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED>
int launch(ds_ctx* ctx, MmArgs& a) {
  const void* x = TRANSPOSED ? a.dy : a.x;
  const int depth = TRANSPOSED ? a.outer : a.inner;
  const bool direct = sixteen(x, TRANSPOSED ? a.dys : a.xs, sizeof(T)) && sixteen(a.w, a.outer, sizeof(T)) && depth % Piece<T>::N == 0;
  return direct ? launch_one<T, BR, BN, WR, WN, TRANSPOSED, true>(ctx, a) : launch_one<T, BR, BN, WR, WN, TRANSPOSED, false>(ctx, a);
}

}  // namespace

int ds_launch_row_tiles(ds_ctx* ctx, int dtype, bool transposed, MmArgs& a) {
  if (dtype == DS_ELEM_F32) return transposed ? launch<float, 128, 128, 2, 2, true>(ctx, a) : launch<float, 128, 128, 2, 2, false>(ctx, a);
  if (dtype == DS_ELEM_BF16) return transposed ? launch<__bf16, 256, 256, 2, 4, true>(ctx, a) : launch<__bf16, 256, 256, 2, 4, false>(ctx, a);
  return transposed ? launch<_Float16, 256, 256, 2, 4, true>(ctx, a) : launch<_Float16, 256, 256, 2, 4, false>(ctx, a);
}

int64_t ds_weight_tiles_bytes(int dtype) {
  const int64_t side = dtype == DS_ELEM_F32 ? 128 : 256;
  return kWeightGroups * 2 * (side * side + side) * (int64_t)sizeof(float);
}

int ds_launch_weight_tiles(ds_ctx* ctx, int dtype, MmArgs& a, void* partial) {
  if (dtype == DS_ELEM_F32) return launch_weights<float, 128, 128, 2, 2>(ctx, a, (float*)partial);
  if (dtype == DS_ELEM_BF16) return launch_weights<__bf16, 256, 256, 2, 4>(ctx, a, (float*)partial);
  return launch_weights<_Float16, 256, 256, 2, 4>(ctx, a, (float*)partial);
}
