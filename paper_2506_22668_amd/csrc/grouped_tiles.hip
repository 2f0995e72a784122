// Products of rows with the weights of their group where a group has many rows: tiles through LDS.
#include "grouped_mm.h"
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

// Brings a step of an operand into LDS: piece u of thread t is piece number u * threads + t of the tile.
template <typename T, int COLS, bool ACROSS, int THREADS, bool DIRECT>
struct Loader {
  using Op = Operand<T, COLS, ACROSS>;
  static constexpr int N = Op::N, PIECES = Op::BYTES / 16 / THREADS;
  const T* from[PIECES];   // of the thread's pieces, at step 0
  int limit[PIECES];       // not ACROSS: the contraction's end, as seen from the piece, or 0 (no such column); ACROSS: elements from the piece's column on
  PieceV<T> held[DIRECT ? 1 : PIECES];

  __device__ __forceinline__ void store(char* tile) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int u = 0; u < PIECES; ++u) *reinterpret_cast<PieceV<T>*>(tile + (u * THREADS + (int)threadIdx.x) * 16) = held[u];
    }
  }
  __device__ __forceinline__ void fetch(int u, const T* p, int have, char* tile) {
    if constexpr (DIRECT) {
      const T* src = have > 0 ? p : reinterpret_cast<const T*>(&kZeros);
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      __builtin_amdgcn_global_load_lds((const DS_GLOBAL void*)src, (DS_LDS void*)(tile + (u * THREADS + wave * 64) * 16), 16, 0, 0);
    } else {
      held[u] = load_piece<T>(p, have);
    }
  }
};

template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WN, 2) void row_tiles_kernel(MmArgs a) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T);
  constexpr int NR = BR / WR / 32, NN = BN / WN / 32, SLICES = DEPTH / (2 * N);
  constexpr int SHIFT = BR == 256 ? 8 : BR == 128 ? 7 : 6;
  using XOp = Operand<T, BR, false>;
  using WOp = Operand<T, BN, !TRANSPOSED>;
  constexpr int STAGE = XOp::BYTES + WOp::BYTES;
  // (two arrays, not halves of one: only then does the compiler know that what is read of one does not wait for what comes into the other)
  __shared__ __attribute__((aligned(128))) char even[STAGE], odd[STAGE];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wr = (wave / WN) * (BR / WR), wn = (wave % WN) * (BN / WN);
  const int width = TRANSPOSED ? a.inner : a.outer, depth = TRANSPOSED ? a.outer : a.inner;
  // Workgroups go to the eight XCDs in turn: each XCD takes a stretch of the tiles, so that the column tiles of a row tile share an L2
  const int per = (int)gridDim.x >> 3;
  const int at = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
  const int tile = at / a.col_tiles, col0 = at % a.col_tiles * BN;
  GroupTile gt;
  if (!find_group_tile(a.offsets, a.groups, a.rows, SHIFT, tile, &gt)) return;
  int row[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int pos = gt.begin + wr + r * 32 + (lane & 31);
    row[r] = pos < gt.end ? ds_ordered_row(a.order, a.rows, pos) : -1;
  }
  f32x16 acc[NR][NN] = {};
  if (gt.group < a.groups) {
    const T* x = (const T*)(TRANSPOSED ? a.dy : a.x);
    const int64_t xs = TRANSPOSED ? a.dys : a.xs;
    const T* w = (const T*)a.w + (int64_t)gt.group * a.inner * a.outer;
    Loader<T, BR, false, THREADS, DIRECT> lx;
    Loader<T, BN, !TRANSPOSED, THREADS, DIRECT> lw;
#pragma unroll
    for (int u = 0; u < lx.PIECES; ++u) {
      const int n = u * THREADS + (int)threadIdx.x, pos = gt.begin + XOp::line(n), k = XOp::piece(n) * N;
      const int r = pos < gt.end ? ds_ordered_row(a.order, a.rows, pos) : -1;
      lx.from[u] = x + (r < 0 ? 0 : r) * xs + k;
      lx.limit[u] = r < 0 ? 0 : depth - k;
    }
#pragma unroll
    for (int u = 0; u < lw.PIECES; ++u) {
      const int n = u * THREADS + (int)threadIdx.x;
      if constexpr (TRANSPOSED) {
        const int col = col0 + WOp::line(n), k = WOp::piece(n) * N;
        lw.from[u] = w + (int64_t)col * a.outer + k;
        lw.limit[u] = col < width ? depth - k : 0;
      } else {
        const int col = col0 + WOp::piece(n) * N;
        lw.from[u] = w + (int64_t)WOp::line(n) * a.outer + col;
        lw.limit[u] = width - col;
      }
    }
    const auto fetch = [&](int k, char* stage) {
#pragma unroll
      for (int u = 0; u < lw.PIECES; ++u) {
        if constexpr (TRANSPOSED) {
          lw.fetch(u, lw.from[u] + k, lw.limit[u] - k, stage);
        } else {
          const int line = WOp::line(u * THREADS + (int)threadIdx.x);
          lw.fetch(u, lw.from[u] + (int64_t)k * a.outer, k + line < depth ? lw.limit[u] : 0, stage);
        }
      }
#pragma unroll
      for (int u = 0; u < lx.PIECES; ++u) lx.fetch(u, lx.from[u] + k, lx.limit[u] - k, stage + WOp::BYTES);
    };
    const Reader<T, BR, false, false> rx(lane);
    const Reader<T, BN, !TRANSPOSED, true> rw(lane);
    const auto compute = [&](const char* stage) {
#pragma unroll
      for (int s = 0; s < SLICES; ++s) {
        PieceV<T> fx[NR], fw[NN];
#pragma unroll
        for (int r = 0; r < NR; ++r) fx[r] = rx.read(stage + WOp::BYTES, wr + r * 32, s);
#pragma unroll
        for (int n = 0; n < NN; ++n) fw[n] = rw.read(stage, wn + n * 32, s);
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int n = 0; n < NN; ++n) acc[r][n] = multiply(fw[n], fx[r], acc[r][n]);
      }
    };
    const int steps = (depth + DEPTH - 1) / DEPTH;
    const auto step = [&](int s, char* now, char* then) {
      __syncthreads();
      if (s + 1 < steps) fetch((s + 1) * DEPTH, then);
      compute(now);
      if (s + 1 < steps) {
        lw.store(then);
        lx.store(then + WOp::BYTES);
      }
    };
    fetch(0, even);
    lw.store(even);
    lx.store(even + WOp::BYTES);
    for (int s = 0; s < steps; s += 2) {
      step(s, even, odd);
      if (s + 1 < steps) step(s + 1, odd, even);
    }
  }
  const T* gate = (const T*)a.gate;
  T* y = (T*)a.y;
#pragma unroll
  for (int n = 0; n < NN; ++n) {
    const int col = col0 + wn + n * 32 + 16 * (lane >> 5);
    float bias[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) bias[i] = a.bias && gt.group < a.groups && col + i < width ? a.bias[(int64_t)gt.group * width + col + i] : 0.f;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      if (row[r] < 0) continue;
#pragma unroll
      for (int p = 0; p < 16 / N; ++p) {
        const int c = col + p * N;
        if (c >= width) continue;
        const PieceV<T> open = gate ? load_piece<T>(gate + row[r] * a.gs + c, width - c) : PieceV<T>{};
        PieceV<T> out;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          float v = acc[r][n][p * N + i] + bias[p * N + i];
          if (a.relu) v = v < 0.f ? 0.f : v;   // (a NaN stays one)
          if (gate) v = (float)open[i] > 0.f ? v : 0.f;
          out[i] = (T)v;
        }
        store_piece<T>(y + row[r] * a.ys + c, out, width - c);
      }
    }
  }
}

template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED, bool DIRECT>
int launch_one(ds_ctx* ctx, MmArgs& a) {
  constexpr int SHIFT = BR == 256 ? 8 : BR == 128 ? 7 : 6;
  a.col_tiles = ((TRANSPOSED ? a.inner : a.outer) + BN - 1) / BN;
  const int64_t tiles = (ds_most_tiles(a, SHIFT) * a.col_tiles + 7) / 8 * 8;
  if (tiles > 0x7fffffff) return ds_fail(ctx, DS_EINVAL, "%d rows by %d columns are more tiles than a launch has", a.rows, TRANSPOSED ? a.inner : a.outer);
  const auto kernel = row_tiles_kernel<T, BR, BN, WR, WN, TRANSPOSED, DIRECT>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(64 * WR * WN), 0, ctx->stream, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

bool sixteen(const void* p, int64_t stride, size_t element) { return (uintptr_t)p % 16 == 0 && stride * element % 16 == 0; }

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
