// Products of rows with the weights of their group where a group has many rows: tiles through LDS.
#include "grouped_mm.h"
#include "mm_split.h"
#include "rows.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define DS_LDS __attribute__((address_space(3)))
#define DS_GLOBAL __attribute__((address_space(1)))


__device__ const uint4 kZeros = {0, 0, 0, 0};

// Part `part` of the product of two pieces: 16-bit ones take one instruction, fp32 ones four (which one after the other would each
// wait for the sum of the last: see products)
template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 4 : 1;
__device__ __forceinline__ f32x16 multiply(PieceV<__bf16> a, PieceV<__bf16> b, f32x16 d, int) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(PieceV<_Float16> a, PieceV<_Float16> b, f32x16 d, int) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, d, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(PieceV<float> a, PieceV<float> b, f32x16 d, int part) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a[part], b[part], d, 0, 0, 0);
}
// all products of a slice, or their parts FIRST .. LAST - 1
template <typename T, int NR, int NN, int FIRST = 0, int LAST = kParts<T>>
__device__ __forceinline__ void products(const PieceV<T> (&fw)[NN], const PieceV<T> (&fx)[NR], f32x16 (&acc)[NR][NN]) {
#pragma unroll
  for (int part = FIRST; part < LAST; ++part)
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int n = 0; n < NN; ++n) acc[r][n] = multiply(fw[n], fx[r], acc[r][n], part);
}

// column of the tile that row m of a matrix-core operand stands for: a lane's 16 results are then 16 neighbours
__device__ __forceinline__ int column_of(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

// A stage of an operand in LDS: DEPTH elements of the contraction (64 bytes of them). ACROSS false: [COLS][DEPTH], the 16-byte pieces of
// a column exchanged by bits of its number; true: [DEPTH][COLS], pieces exchanged by the step's last two bits (16-bit types). Either way
// the lanes that read together meet all banks.
constexpr int kDepthBytes = 64;
template <typename T, int COLS, bool ACROSS>
struct Operand {
  static constexpr int N = Piece<T>::N, BYTES = COLS * kDepthBytes;
  static constexpr int PER_ROW = ACROSS ? COLS / N : kDepthBytes / 16;
  static __device__ __forceinline__ int exchange(int line, int piece) {
    if constexpr (ACROSS) return sizeof(T) == 2 ? piece ^ ((line & 3) << 2) : piece;
    else return piece ^ ((line >> 1) & 3);
  }
  // the place of piece number `at` of the stage: its column (or step) and which piece of that
  static __device__ __forceinline__ int line(int at) { return at / PER_ROW; }
  static __device__ __forceinline__ int piece(int at) { return exchange(line(at), at % PER_ROW); }
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
  // columns first .. first + 31 (first: a multiple of 32), steps slice * 2 N ..
  __device__ __forceinline__ PieceV<T> read(const char* stage, int first, int slice) const {
    constexpr int N = Op::N;
    if constexpr (!ACROSS) {
      return *reinterpret_cast<const PieceV<T>*>(stage + (first + m) * kDepthBytes + (Op::exchange(m, 2 * slice + h) << 4));
    } else if constexpr (sizeof(T) == 2) {
      const int i = lane & 15, four = ((lane >> 4) & 1) * 4 + (i & 3);
      const int col = first + (ORDERED ? 16 * (four & 1) + 4 * (four >> 1) : 4 * four);
      const int byte = (slice * 16 + 8 * h + (i >> 2)) * (COLS * 2) + (Op::exchange(i >> 2, col >> 3) << 4) + (col & 7) * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DS_LDS s16x4*)(stage + byte));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DS_LDS s16x4*)(stage + byte + 4 * COLS * 2));
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
        v[i] = *reinterpret_cast<const float*>(stage + (slice * 2 * N + N * h + i) * (COLS * 4) + (first + m) * 4);
      return v;
    }
  }
};

// Brings pieces of an operand into LDS: piece u of thread t is piece number u * THREADS + t of the stage. Direct loads go there by themselves;
// rows that are not aligned for them come through registers.
template <typename T, int STAGE_BYTES, int THREADS, bool DIRECT>
struct Loader {
  static constexpr int N = Piece<T>::N, PIECES = STAGE_BYTES / 16 / THREADS;
  PieceV<T> held[DIRECT ? 1 : PIECES];
  unsigned over = 0;   // four bits a piece: by how many elements it would reach over the matrix' end

  // The piece at p, zeros if it is not `there`. Where columns end in it, what lies behind them comes along: the next row's, or what is between
  // the rows, up to the matrix' `end`; it meets results only that nobody stores. (edge: whether any lane's piece may not be there
  // or may reach over the end. One that would is read so that it ends there, and shifted on its way into LDS.)
  __device__ __forceinline__ void fetch(int u, const T* p, bool there, bool edge, const T* end, char* stage) {
    const T* zeros = reinterpret_cast<const T*>(&kZeros);
    if constexpr (DIRECT) {   // (rows are whole pieces)
      const T* src = there && p < end ? p : zeros;
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      __builtin_amdgcn_global_load_lds((const DS_GLOBAL void*)src, (DS_LDS void*)(stage + (u * THREADS + wave * 64) * 16), 16, 0, 0);
    } else {
      if (u == 0) over = 0;
      if (edge) {
        const int64_t by = there ? p + N - end : 0;
        over |= (unsigned)(by <= 0 ? 0 : by < N ? by : N) << (4 * u);
        p = !there ? zeros : by > 0 ? end - N : p;
      }
      held[u] = *reinterpret_cast<const typename Piece<T>::U*>(p);
    }
  }
  // into LDS; cut: of each piece its first `keep` elements alone (the contraction ends in it)
  __device__ __forceinline__ void store(char* stage, bool cut, int keep) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int u = 0; u < PIECES; ++u) {
        if (__any(over >> (4 * u) & 15)) held[u] = shifted<T>(held[u], over >> (4 * u) & 15);
        if (cut) held[u] = first_elements<T>(held[u], keep);
        *reinterpret_cast<PieceV<T>*>(stage + (u * THREADS + (int)threadIdx.x) * 16) = held[u];
      }
    }
  }
};

constexpr int kMostGroups = 1024;

// Tiles up to the last of every group, in LDS: a tile's group is found by two ballots
struct GroupTable {
  int upto[kMostGroups], waves[16];
};

// Fills the table (all threads of the workgroup); the number of tiles
template <int THREADS, int SHIFT>
__device__ __forceinline__ int fill_table(GroupTable& t, const MmArgs& a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, most = ds_most_parts(a.rows, 1 << SHIFT, a.groups + 1);
  int before = 0;
  for (int base = 0; base < kMostGroups; base += THREADS) {
    const int g = base + (int)threadIdx.x;
    if (base >= a.groups) {
      t.upto[g] = before;
      continue;
    }
    int begin = 0, end = 0;
    if (g < a.groups) ds_group_range(a.offsets, a.groups, a.rows, g, &begin, &end);
    int upto = ds_parts_of(begin, end, 1 << SHIFT);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(upto, o, 64);
      if (lane >= o) upto = ds_add_parts(upto, up, most);
    }
    if (lane == 63) t.waves[wave] = upto;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) upto = ds_add_parts(upto, t.waves[w], most);
      all = ds_add_parts(all, t.waves[w], most);
    }
    t.upto[g] = ds_add_parts(before, upto, most);
    before = ds_add_parts(before, all, most);
    __syncthreads();
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(before);
}

// Tile `tile` (one that there is); the same answer in every lane
template <int SHIFT>
__device__ __forceinline__ GroupTile find_tile(const GroupTable& t, const MmArgs& a, int tile) {
  const int lane = threadIdx.x & 63;
  const int sixteen = __ffsll((long long)__ballot(t.upto[lane * 16 + 15] > tile)) - 1;
  const int g = __builtin_amdgcn_readfirstlane(sixteen * 16 + __ffsll((long long)__ballot(t.upto[sixteen * 16 + (lane & 15)] > tile)) - 1);
  int begin, end;
  ds_group_range(a.offsets, a.groups, a.rows, g, &begin, &end);
  begin += (tile - (g ? t.upto[g - 1] : 0)) << SHIFT;
  GroupTile out;
  out.group = g;
  out.begin = __builtin_amdgcn_readfirstlane(begin);
  out.end = __builtin_amdgcn_readfirstlane(min(end, begin + (1 << SHIFT)));
  return out;
}

// Waits until all but the last LATER of the wave's loads and stores are done (-1: without that), then for the workgroup's other waves:
// what they brought into LDS is there. (A plain barrier waits for LDS accesses, but not for loads that go to LDS directly.)
template <int LATER>
__device__ __forceinline__ void meet() {
  if constexpr (LATER >= 0) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LATER) : "memory");
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The same value, of which the compiler knows nothing: what is computed from it stays where it stands, out of the registers of a loop around it.
__device__ __forceinline__ int hidden(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Workgroups stay: one to a compute unit (of 256 threads: two), which goes through tiles of BR rows and BN columns as through one line of steps of the
// contraction (128 bytes of every row). A step is computed on from one half of the LDS, the next one is in the other half already, and
// what comes behind that, of this tile or the next, is asked for as soon as the first half is through; a wave's operands for a slice of the
// step are read while the matrix cores work on the slice before. Results leave through LDS of their own, while the next tile's steps come in.
// Long contractions are bound by the matrix cores and the card's power (65,536 rows by 4,096 x 1,024 bf16 in 8 groups 602 us, 910 TFLOP/s; a large
// library product 1,218), short ones by the results, which no products go on beside (a unit has the registers of one such tile), and by the last
// round of tiles: 131,072 rows by 1,024 x 1,024, rows gathered and scattered, 340 us, 810 TFLOP/s; dx of 65,521 rows by 1,024 x 512 with its gate 150 us,
// 460 TFLOP/s, 2.2 TB/s; fp32 30,011 rows by 512 x 256 76 us, 104 TFLOP/s (a large library product: 153).
template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WN, 2) void row_tiles_kernel(MmArgs a) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T);
  constexpr int TR = BR / WR, TN = BN / WN, NR = TR / 32, NN = TN / 32, SLICES = DEPTH / (2 * N);
  constexpr int SHIFT = BR == 256 ? 8 : 7;
  using XOp = Operand<T, BR, false>;
  using WOp = Operand<T, BN, !TRANSPOSED>;
  constexpr int STAGE = XOp::BYTES + WOp::BYTES, LOADS = STAGE / 16 / THREADS;
  constexpr int OUT_ROW = TN * (int)sizeof(T), CHUNKS = OUT_ROW / 16, AT_ONCE = 64 / CHUNKS, OUT_ROWS = 16, OUTS = OUT_ROWS / AT_ONCE;
  // (arrays, not parts of one: only then does the compiler know that what is read of one does not wait for what comes into the other)
  __shared__ __attribute__((aligned(128))) char stage0[STAGE], stage1[STAGE], stage2[STAGE], stage3[STAGE], leaving[WR * WN * OUT_ROWS * OUT_ROW];
  __shared__ __attribute__((aligned(16))) float bias_of[WR * WN * TN];
  __shared__ GroupTable table;
  // of the tiles under way, by their number: the rows, and the group (a tile comes in at most four or, fp32, five stages before it is computed on,
  // and has two at the least: three or four tiles are under way)
  constexpr int HELD = sizeof(T) == 2 ? 4 : 8;
  __shared__ int row_of[HELD][BR], group_of[HELD];
  static_assert(sizeof(stage0) * 4 + sizeof(leaving) + sizeof(bias_of) + sizeof(table) + sizeof(row_of) + sizeof(group_of) <= (THREADS == 256 ? 80 : 160) * 1024, "");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (wave / WN) * TR, wn = (wave % WN) * TN;
  const int width = TRANSPOSED ? a.inner : a.outer, depth = TRANSPOSED ? a.outer : a.inner;
  const T* x = (const T*)(TRANSPOSED ? a.dy : a.x);
  const int64_t xs = TRANSPOSED ? a.dys : a.xs;
  const T *gate = (const T*)a.gate, *gate_end = gate + (int64_t)(a.rows - 1) * a.gs + width;
  T* y = (T*)a.y;
  // Workgroups go to the eight XCDs in turn. Each XCD has a stretch of the tiles, column tiles of a row tile next to each other, so that they
  // share its L2; its workgroups take them in turn.
  const int64_t tiles = (int64_t)fill_table<THREADS, SHIFT>(table, a) * a.col_tiles;
  const int xcd = (int)blockIdx.x & 7, step_by = (int)gridDim.x >> 3;
  const int stretch = __builtin_amdgcn_readfirstlane((int)(tiles * (xcd + 1) / 8));
  int at = __builtin_amdgcn_readfirstlane((int)(tiles * xcd / 8) + ((int)blockIdx.x >> 3));

  Loader<T, XOp::BYTES, THREADS, DIRECT> lx;
  Loader<T, WOp::BYTES, THREADS, DIRECT> lw;
  const T *x_end = x + (int64_t)(a.rows - 1) * xs + depth, *w_end = (const T*)a.w + (int64_t)a.groups * a.inner * a.outer;
  const Reader<T, BR, false, false> rx(lane);
  const Reader<T, BN, !TRANSPOSED, true> rw(lane);
  const int steps = (depth + 2 * DEPTH - 1) / (2 * DEPTH) * 2;   // stages of a tile, an even number (zeros behind the end)
  // A thread's pieces of a step lie in one place of lines that are a fixed number apart (the exchange of pieces goes by the last bits
  // of a line, which that number leaves alone)
  constexpr int XLINES = THREADS / XOp::PER_ROW, WLINES = THREADS / WOp::PER_ROW;
  static_assert(XLINES % 8 == 0 && WLINES % 8 == 0, "");
  const int xk = XOp::piece((int)threadIdx.x) * N;
  const int wline = WOp::line((int)threadIdx.x), wplace = WOp::piece((int)threadIdx.x) * N;
  // what comes in: step `coming` of the tile `coming_at`, whose rows were looked up while the tile before came in
  const T *from_x[lx.PIECES], *from_w;
  int row[lx.PIECES], coming = 0, coming_col = 0, coming_at = at, coming_group = 0, coming_number = 0;
  const auto look_up = [&](int tile) __attribute__((always_inline)) {
    const GroupTile found = find_tile<SHIFT>(table, a, tile / a.col_tiles);
    coming_group = found.group;
    const int line = XOp::line(hidden((int)threadIdx.x));
#pragma unroll
    for (int u = 0; u < lx.PIECES; ++u) {
      const int pos = found.begin + u * XLINES + line;
      row[u] = pos < found.end ? ds_ordered_row(a.order, a.rows, pos) : -1;
    }
  };
  // Asks for the next stage: number `coming` of tile `coming_at`; behind the last one nothing (false).
  const auto fetch = [&](char* stage) __attribute__((always_inline)) {
    if (coming_at >= stretch) return false;
    if (coming == 0) {
      coming_col = coming_at % a.col_tiles * BN;
      from_w = (const T*)a.w + (int64_t)coming_group * a.inner * a.outer +
               (TRANSPOSED ? (int64_t)(coming_col + wline) * a.outer + wplace : (int64_t)wline * a.outer + coming_col + wplace);
      int* rows = row_of[coming_number & (HELD - 1)];
      const int tid = hidden((int)threadIdx.x);
#pragma unroll
      for (int u = 0; u < lx.PIECES; ++u) {
        from_x[u] = x + (row[u] < 0 ? 0 : row[u]) * xs + xk;   // (no row: any row, whose results go nowhere)
        if (tid % XOp::PER_ROW == 0) rows[u * XLINES + XOp::line(tid)] = row[u];
      }
      group_of[coming_number & (HELD - 1)] = coming_group;
      ++coming_number;
      if (coming_at + step_by < stretch) look_up(coming_at + step_by);
    }
    const int k = coming * DEPTH;
    const bool deep = k + DEPTH > depth, wide = coming_col + BN > width;
#pragma unroll
    for (int u = 0; u < lx.PIECES; ++u) lx.fetch(u, from_x[u] + k, k + xk < depth, deep, x_end, stage + WOp::BYTES);
#pragma unroll
    for (int u = 0; u < lw.PIECES; ++u) {
      const int line = u * WLINES + wline;
      if constexpr (TRANSPOSED)
        lw.fetch(u, from_w + (int64_t)(u * WLINES) * a.outer + k, coming_col + line < width && k + wplace < depth, deep || wide, w_end, stage);
      else lw.fetch(u, from_w + (int64_t)(k + u * WLINES) * a.outer, k + line < depth, deep || wide, w_end, stage);
    }
    if (++coming == steps) {
      coming = 0;
      coming_at += step_by;
    }
    return true;
  };
  // what came through registers: the stage that was asked for last
  const auto put = [&](char* stage) __attribute__((always_inline)) {
    const int k = ((coming == 0 ? steps : coming) - 1) * DEPTH;
    lw.store(stage, TRANSPOSED && k + DEPTH > depth, depth - k - wplace);
    lx.store(stage + WOp::BYTES, k + DEPTH > depth, depth - k - xk);
  };

  if (at < stretch) {
    f32x16 acc[NR][NN] = {};
    PieceV<T> fx[2][NR], fw[2][NN];
    const auto read = [&](const char* stage, int c) __attribute__((always_inline)) {
#pragma unroll
      for (int n = 0; n < NN; ++n) fw[c & 1][n] = rw.read(stage, wn + n * 32, c);
#pragma unroll
      for (int r = 0; r < NR; ++r) fx[c & 1][r] = rx.read(stage + WOp::BYTES, wr + r * 32, c);
    };
    // One stage.
    // PAIRED (16-bit types): in two phases between barriers, the wave's operands out of LDS and loads of what comes three stages on, into the stage
    // that was `before`; then nothing but products. The two waves of a SIMD are a phase apart, so that one fills the matrix cores while
    // the other works off addresses and waits.
    // Otherwise (fp32, whose products take 16 times as long): operands of a slice are read under the products of the one before, and loads of
    // what comes four stages on are asked for, into `now`, where nobody reads it any more; one barrier. (65,536 rows by 512 x 512: 0.39 ms in phases.)
    // Waits leave the loads of two stages under way (near the end, where there are no more, none). `fresh`: in the two stages
    // behind a tile's results, in front of whose stores all loads were waited for, so that the stores need not be.
    constexpr bool PAIRED = sizeof(T) == 2;
    const auto half = [&](bool fresh, bool last, char* before, char* now, char* then) __attribute__((always_inline)) {
      if constexpr (PAIRED) {
        read(now, 0);
        read(now, 1);
        put(before);
        const bool more = fetch(before);
        if (!DIRECT || fresh) meet<-1>();
        else if (more) meet<2 * LOADS>();
        else meet<0>();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
        products<T, NR, NN>(fw[0], fx[0], acc);
        products<T, NR, NN>(fw[1], fx[1], acc);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        meet<-1>();
      } else {
        read(now, 1);
        __builtin_amdgcn_sched_barrier(0);
        products<T, NR, NN>(fw[0], fx[0], acc);
        __builtin_amdgcn_sched_barrier(0);
        if (!DIRECT || fresh) meet<-1>();
        else if (coming_at < stretch) meet<2 * LOADS>();
        else meet<0>();
        if (!last) read(then, 0);
        __builtin_amdgcn_sched_barrier(0);
        products<T, NR, NN, 0, kParts<T> / 2>(fw[1], fx[1], acc);
        __builtin_amdgcn_sched_barrier(0);
        put(now);
        fetch(now);
        __builtin_amdgcn_sched_barrier(0);
        products<T, NR, NN, kParts<T> / 2, kParts<T>>(fw[1], fx[1], acc);
      }
    };
    static_assert(SLICES == 2, "");
    int number = 0;
    const auto leave = [&]() __attribute__((always_inline)) {
      const int lane = hidden((int)threadIdx.x & 63), col = at % a.col_tiles * BN + wn;
      char* mine = leaving + wave * (OUT_ROWS * OUT_ROW);
      float* bias = bias_of + wave * TN;
      if constexpr (!TRANSPOSED) {
        const float* from = a.bias + (a.bias ? (int64_t)__builtin_amdgcn_readfirstlane(group_of[number & (HELD - 1)]) * width : 0);
#pragma unroll
        for (int j = 0; j < TN; j += 64)
          if (TN % 64 == 0 || j + lane < TN) bias[j + lane] = a.bias ? from[min(col + j + lane, width - 1)] : 0.f;
      }
      const float least = !TRANSPOSED && a.relu ? 0.f : -INFINITY;
      const int chunk = lane % CHUNKS, c = col + chunk * N;
      const int* rows = row_of[number & (HELD - 1)] + wr + lane / CHUNKS;
      // (a gate is asked for two blocks of rows ahead, in front of stores that its coming would otherwise wait for)
      PieceV<T> open[2 * NR][OUTS];
      const auto ask = [&](int r) __attribute__((always_inline)) {
        if constexpr (TRANSPOSED) {
          if (gate && r < NR) {
#pragma unroll
            for (int half = 2 * r; half < 2 * r + 2; ++half)
#pragma unroll
              for (int i = 0; i < OUTS; ++i) {
                const int to = rows[half * OUT_ROWS + i * AT_ONCE];
                if (to >= 0 && c < width) open[half][i] = load_within<T>(gate + to * a.gs + c, gate_end);
              }
          }
        }
      };
      ask(0);
      ask(1);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the next step has come in: see step)
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        PieceV<T> out[NN][16 / N];
#pragma unroll
        for (int n = 0; n < NN; ++n)
#pragma unroll
          for (int p = 0; p < 16 / N; ++p)
#pragma unroll
            for (int q = 0; q < N; q += 4) {
              float4 b = {0.f, 0.f, 0.f, 0.f};
              if constexpr (!TRANSPOSED) b = *reinterpret_cast<const float4*>(bias + n * 32 + 16 * (lane >> 5) + p * N + q);
              const float plus[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float v = acc[r][n][p * N + q + i];
                if constexpr (!TRANSPOSED) {
                  v += plus[i];
                  v = v < least ? least : v;   // (a NaN stays one)
                }
                out[n][p][q + i] = (T)v;
              }
            }
        if (r) ask(r + 1);
#pragma unroll
        for (int h = 0; h < 2; ++h) {   // 16 rows at a time
          const int half = 2 * r + h;
          if (((lane >> 4) & 1) == h) {
#pragma unroll
            for (int n = 0; n < NN; ++n)
#pragma unroll
              for (int p = 0; p < 16 / N; ++p)
                *reinterpret_cast<PieceV<T>*>(mine + (lane & 15) * OUT_ROW + ((((n * 32 + 16 * (lane >> 5)) / N + p) ^ (lane & 7)) << 4)) = out[n][p];
          }
          // (a wave reads what it wrote itself: its LDS accesses keep their order)
#pragma unroll
          for (int i = 0; i < OUTS; ++i) {
            const int line = i * AT_ONCE + lane / CHUNKS, to = rows[half * OUT_ROWS + i * AT_ONCE];
            const char* held = mine + line * OUT_ROW + ((chunk ^ (line & 7)) << 4);
            if (to < 0 || c >= width) continue;
            PieceV<T> v = *reinterpret_cast<const PieceV<T>*>(held);
            if (TRANSPOSED && gate) {
#pragma unroll
              for (int j = 0; j < N; ++j) v[j] = (float)open[half][i][j] > 0.f ? v[j] : (T)0.f;
            }
            T* target = y + to * a.ys + c;
            if (c + N <= width) *reinterpret_cast<typename Piece<T>::U*>(target) = v;
            else store_first<T>(target, v, width - c);
          }
        }
      }
      ++number;
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int n = 0; n < NN; ++n) acc[r][n] = f32x16{};
    };
    look_up(at);
    fetch(stage0);
    put(stage0);
    fetch(stage1);
    put(stage1);
    fetch(stage2);
    put(stage2);
    if (!PAIRED) {
      fetch(stage3);
      put(stage3);
    }
    if (!DIRECT) fetch(PAIRED ? stage3 : stage0);
    meet<0>();
    const bool second = PAIRED && wave >= WR * WN / 2;   // the waves that are a phase behind; all leave a tile together
    if (second) meet<-1>();
    if (!PAIRED) read(stage0, 0);
    int s = 0;
    bool left = true;
    const auto two = [&](char* before, char* now, char* then, char* behind) __attribute__((always_inline)) {
      s += 2;
      half(left, false, before, now, then);
      half(left, s == steps, now, then, behind);
      left = s == steps;
      if (left) {
        if (PAIRED && !second) meet<-1>();
        leave();
        s = 0;
        at += step_by;
        if (at >= stretch) return false;
        if (second) meet<-1>();
        if (!PAIRED) read(behind, 0);
      }
      return true;
    };
    while (two(stage3, stage0, stage1, stage2) && two(stage1, stage2, stage3, stage0)) {
    }
  }
  // rows of no group
  int none, end;
  ds_group_range(a.offsets, a.groups, a.rows, a.groups, &none, &end);
  for (int pos = none + (int)blockIdx.x * WR * WN + wave; pos < end; pos += (int)gridDim.x * WR * WN) {
    const int r = ds_ordered_row(a.order, a.rows, pos);
    if (r >= 0)
      for (int c = lane * N; c < width; c += 64 * N) store_piece<T>(y + r * a.ys + c, PieceV<T>{}, width - c);
  }
}

template <typename T, int BR, int BN, int WR, int WN, bool TRANSPOSED, bool DIRECT>
int launch_one(ds_ctx* ctx, MmArgs& a) {
  a.col_tiles = ((TRANSPOSED ? a.inner : a.outer) + BN - 1) / BN;
  if (ds_most_tiles(a, BR == 256 ? 8 : 7) * a.col_tiles > 0x7fffffff)
    return ds_fail(ctx, DS_EINVAL, "%d rows by %d columns are more tiles than are counted", a.rows, TRANSPOSED ? a.inner : a.outer);
  constexpr int A_UNIT = WR * WN == 4 ? 2 : 1;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(row_tiles_kernel<T, BR, BN, WR, WN, TRANSPOSED, DIRECT>), dim3((unsigned)(A_UNIT * ctx->num_cus + 7) / 8 * 8),
                     dim3(64 * WR * WN), 0, ctx->stream, a);
  DS_HIP(ctx, hipGetLastError());
  return DS_OK;
}

bool sixteen(const void* p, int64_t stride, size_t element) { return (uintptr_t)p % 16 == 0 && stride * element % 16 == 0; }

// ---- the gradient of the weights ------------------------------------------------------------------------------------------------
// dW_g = sum_r x[r]^T dy[r]: both operands run across the contraction, which is the group's rows. Groups are ragged, and there are about
// as many tiles as compute units or fewer, so the steps of all groups (UNIT rows each) lie in one line that is cut evenly into chunks, and a
// workgroup takes one tile of the weights through one chunk. The tiles of a chunk run beside each other on one XCD and read the same rows: with
// the steps of a tile in one line instead, neighbours read different rows, and all of them came from memory.
// Where a cut falls inside a group, the chunks on both sides leave fp32 sums (at most two a workgroup), which a second launch
// adds up in order: no atomics, the same bits every time. Bound by the matrix cores where groups are long (65,521 rows by 1,024 x 512 bf16 in 16
// groups: 101 us, 680 TFLOP/s) with what begins and ends each cut, and 23 us for adding up 100 MB of sums.
// the steps of a group's contraction
__device__ __forceinline__ int group_steps(const MmArgs& a, int g, int depth, int* begin, int* end) {
  ds_group_range(a.offsets, a.groups, a.rows, g, begin, end);
  return ds_parts_of(*begin, *end, depth);
}

// Steps of all groups, and where step `unit` of the line falls: its group (-1: behind the end) and the steps before it there. Called by whole
// waves, the same answer in every lane.
__device__ __forceinline__ int locate_unit(const MmArgs& a, int depth, int unit, int* group, int* within) {
  const int lane = threadIdx.x & 63, most = ds_most_parts(a.rows, depth, a.groups);
  int before = 0;
  *group = -1;
  for (int base = 0; base < a.groups; base += 64) {
    int begin, end;
    const int g = base + lane, own = g < a.groups ? group_steps(a, g, depth, &begin, &end) : 0;
    int upto = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(upto, o, 64);
      if (lane >= o) upto = ds_add_parts(upto, up, most);
    }
    upto = ds_add_parts(before, upto, most);
    const unsigned long long reach = __ballot(upto > unit);
    if (reach && *group < 0) {
      const int src = __builtin_amdgcn_readfirstlane(__ffsll((long long)reach) - 1);
      *group = base + src;
      *within = unit - __builtin_amdgcn_readlane(upto - own, src);
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return before;
}

template <typename T, int BR, int BN, int WR, int WN, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WN, 2) void weight_tiles_kernel(MmArgs a, float* partial, int most_chunks) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, DEPTH = kDepthBytes / sizeof(T), UNIT = 2 * DEPTH;   // rows of a stage, and of a unit
  constexpr int NR = BR / WR / 32, NN = BN / WN / 32, SLOT = BR * BN + BN;
  using XOp = Operand<T, BR, true>;
  using DOp = Operand<T, BN, true>;
  constexpr int STAGE = XOp::BYTES + DOp::BYTES, LOADS = STAGE / 16 / THREADS;
  constexpr int LINES = THREADS / DOp::PER_ROW, EACH = DEPTH / LINES;   // of a thread's pieces of a stage: lines apart, and how many
  __shared__ __attribute__((aligned(128))) char stage0[STAGE], stage1[STAGE], stage2[STAGE], stage3[STAGE];
  __shared__ float sums[LINES][BN];
  __shared__ int row_of[2][THREADS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (wave / WN) * (BR / WR), wn = (wave % WN) * (BN / WN);
  const int tiles = (a.inner + BR - 1) / BR * a.col_tiles;
  // Workgroups go to the eight XCDs in turn: each XCD has a stretch of the (chunk, tile) pairs
  const int place_of = ((int)blockIdx.x & 7) * ((int)gridDim.x >> 3) + ((int)blockIdx.x >> 3);
  const int chunk = place_of / tiles, tile = place_of % tiles;
  int group, within, none;
  const int units = locate_unit(a, UNIT, 0, &none, &within), chunks = min(units, most_chunks);   // (no chunk without a step)
  if (chunk >= chunks) return;
  int unit = (int)ds_mm_even_begin(chunk, chunks, units);
  const int last = (int)ds_mm_even_begin(chunk + 1, chunks, units);
  locate_unit(a, UNIT, unit, &group, &within);
  const int in0 = tile / a.col_tiles * BR, col0 = tile % a.col_tiles * BN;
  const T *x = (const T*)a.x, *dy = (const T*)a.dy;
  const T *x_end = x + (int64_t)(a.rows - 1) * a.xs + a.inner, *dy_end = dy + (int64_t)(a.rows - 1) * a.dys + a.outer;
  const Reader<T, BR, true, false> rx(lane);
  const Reader<T, BN, true, true> rd(lane);
  static_assert(BR == BN && LINES % 4 == 0, "both operands' pieces of a thread lie in the same rows");
  const int line = DOp::line((int)threadIdx.x), place = DOp::piece((int)threadIdx.x) * N;
  while (unit < last && group < a.groups) {
    int begin, end;
    const int steps = group_steps(a, group, UNIT, &begin, &end);
    if (within >= steps) {   // on to the next group
      ++group;
      within = 0;
      continue;
    }
    const int first = __builtin_amdgcn_readfirstlane(within);
    const int upto = __builtin_amdgcn_readfirstlane(min(first + last - unit, steps));
    f32x16 acc[NR][NN] = {};
    float sum[N] = {};
    Loader<T, XOp::BYTES, THREADS, DIRECT> lx;
    Loader<T, DOp::BYTES, THREADS, DIRECT> ld;
    // The next stage to come in starts at position `coming` of the order, up to `stop`. Its rows are in LDS: THREADS of them come there at once, a
    // block ahead (looked up stage by stage, a line of the order a stage, each stage waited for memory: 150 us where sorted rows took 95).
    const int stop = __builtin_amdgcn_readfirstlane(min(end, begin + upto * UNIT)), stages = 2 * (upto - first);
    const int start = __builtin_amdgcn_readfirstlane(begin + first * UNIT);
    int coming = start, left = stages;
    const auto row_at = [&](int pos) __attribute__((always_inline)) { return pos < stop ? ds_ordered_row(a.order, a.rows, pos) : -1; };
    row_of[0][threadIdx.x] = row_at(start + (int)threadIdx.x);
    int later = row_at(start + THREADS + (int)threadIdx.x);
    __syncthreads();
    const bool ends = a.outer - col0 < BN || a.inner - in0 < BR;   // (columns that there are not)
    const auto fetch = [&](char* stage) __attribute__((always_inline)) {
      if (left == 0) return false;
      const int block = (coming - start) / THREADS, at = (coming - start) % THREADS;
      if (at == 0) {   // (nobody reads the block before any more)
        row_of[(block + 1) & 1][threadIdx.x] = later;
        later = row_at(start + (block + 2) * THREADS + (int)threadIdx.x);
      }
      int now[EACH];
#pragma unroll
      for (int u = 0; u < EACH; ++u) now[u] = row_of[block & 1][at + u * LINES + line];
      const bool over = ends || coming + DEPTH > stop || a.order;   // (an order may name rows that there are not)
#pragma unroll
      for (int u = 0; u < EACH; ++u) ld.fetch(u, dy + now[u] * a.dys + (col0 + place), now[u] >= 0, over, dy_end, stage);
#pragma unroll
      for (int u = 0; u < EACH; ++u) lx.fetch(u, x + now[u] * a.xs + (in0 + place), now[u] >= 0, over, x_end, stage + DOp::BYTES);
      coming += DEPTH;
      --left;
      return true;
    };
    const auto put = [&](char* stage) __attribute__((always_inline)) {
      ld.store(stage, false, 0);
      lx.store(stage + DOp::BYTES, false, 0);
    };
    // (in two phases, the waves of a SIMD a phase apart, as in row_tiles_kernel)
    const auto half = [&](bool fresh, char* now, char* before) __attribute__((always_inline)) {
      PieceV<T> fx[2][NR], fd[2][NN];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int n = 0; n < NN; ++n) fd[c][n] = rd.read(now, wn + n * 32, c);
#pragma unroll
        for (int r = 0; r < NR; ++r) fx[c][r] = rx.read(now + DOp::BYTES, wr + r * 32, c);
      }
      if (in0 == 0) {   // db: the column sums of what is in LDS anyway
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
          const PieceV<T> v = *reinterpret_cast<const PieceV<T>*>(now + (u * THREADS + (int)threadIdx.x) * 16);
#pragma unroll
          for (int i = 0; i < N; ++i) sum[i] += (float)v[i];
        }
      }
      put(before);
      const bool more = fetch(before);
      if (!DIRECT || fresh) meet<-1>();
      else if (more) meet<2 * LOADS>();
      else meet<0>();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      products<T, NR, NN>(fd[0], fx[0], acc);
      products<T, NR, NN>(fd[1], fx[1], acc);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
      meet<-1>();
    };
    fetch(stage0);
    put(stage0);
    fetch(stage1);
    put(stage1);
    fetch(stage2);
    put(stage2);
    if (!DIRECT) fetch(stage3);
    meet<0>();
    const bool second = wave >= WR * WN / 2;
    if (second) meet<-1>();
    for (int s = 0; s < stages; s += 4) {
      half(s == 0, stage0, stage3);
      half(s == 0, stage1, stage0);
      if (s + 2 < stages) {
        half(false, stage2, stage1);
        half(false, stage3, stage2);
      }
    }
    if (!second) meet<-1>();
    const bool whole = first == 0 && upto == steps;
    // slot 0: the group began in an earlier chunk; 1: it begins here and goes on in a later one
    float* to = partial + ((int64_t)place_of * 2 + (first == 0)) * SLOT;
    if (in0 == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) sums[line][place + i] = sum[i];
      __syncthreads();
      if (threadIdx.x < BN) {
        float v = 0.f;
#pragma unroll
        for (int p = 0; p < LINES; ++p) v += sums[p][threadIdx.x];
        if (!whole) to[BR * BN + threadIdx.x] = v;
        else if (col0 + (int)threadIdx.x < a.outer) a.db[(int64_t)group * a.outer + col0 + threadIdx.x] = v;
      }
      __syncthreads();
    }
    if (whole) {
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
    } else {
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int n = 0; n < NN; ++n)
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const float4 v = {acc[r][n][4 * p], acc[r][n][4 * p + 1], acc[r][n][4 * p + 2], acc[r][n][4 * p + 3]};
            reinterpret_cast<float4*>(to)[((r * NN + n) * 4 + p) * THREADS + threadIdx.x] = v;
          }
    }
    unit += upto - first;
    within += upto - first;
  }
}

constexpr int kJoin = 512;   // threads of a workgroup that adds up

// Adds up the sums of groups that were cut, and clears the gradients of empty ones. 16 neighbouring results of a lane of the tile's workgroup are
// a unit; `lanes` threads share a unit's chunks (each takes every lanes-th, and their sums meet in LDS, in order), `parts` workgroups a tile.
template <typename T, int BR, int BN, int WR, int WN>
__global__ __launch_bounds__(kJoin) void weight_join_kernel(MmArgs a, const float* partial, int most_chunks, int parts, int lanes) {
  constexpr int THREADS = 64 * WR * WN, N = Piece<T>::N, UNIT = 128 / sizeof(T);
  constexpr int NR = BR / WR / 32, NN = BN / WN / 32, SLOT = BR * BN + BN;
  __shared__ float4 meet[4][kJoin];
  const int tiles = (a.inner + BR - 1) / BR * a.col_tiles;
  const int group = (int)blockIdx.y, tile = (int)blockIdx.x / parts, part = (int)blockIdx.x % parts;
  const int in0 = tile / a.col_tiles * BR, col0 = tile % a.col_tiles * BN;
  int begin, end;
  const int steps = group_steps(a, group, UNIT, &begin, &end);
  int first = 0, last = -1;
  if (steps > 0) {
    // where the group's steps lie in the line: those of the groups before it first
    const int most = ds_most_parts(a.rows, UNIT, a.groups);
    int mine = 0, all = 0;
    for (int g = threadIdx.x & 63; g < a.groups; g += 64) {
      int b, e;
      const int own = group_steps(a, g, UNIT, &b, &e);
      all = ds_add_parts(all, own, most);
      if (g < group) mine = ds_add_parts(mine, own, most);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      all = ds_add_parts(all, __shfl_xor(all, o, 64), most);
      mine = ds_add_parts(mine, __shfl_xor(mine, o, 64), most);
    }
    const int chunks = min(all, most_chunks);
    ds_group_owners(mine, steps, all, [&](int step) { return (int)ds_mm_even_owner(step, chunks, all); }, &first, &last);
    if (first == last) return;
  }
  const int across = kJoin / lanes, at = (int)threadIdx.x % across, turn = (int)threadIdx.x / across;
  const auto sums = [&](int b) { return partial + (((int64_t)b * tiles + tile) * 2 + (b == first)) * SLOT; };
  T* dw = (T*)a.dw + (int64_t)group * a.inner * a.outer;
  const int units = NR * NN * THREADS, each = (units + parts - 1) / parts, stop = min(units, (part + 1) * each);
  for (int base = part * each; base < stop; base += across) {
    const int unit = base + at, block = unit / THREADS, thread = unit % THREADS, lane = thread & 63, wave = thread >> 6;
    const int in = in0 + wave / WN * (BR / WR) + block / NN * 32 + (lane & 31);
    const int col = col0 + wave % WN * (BN / WN) + block % NN * 32 + 16 * (lane >> 5);
    const bool there = unit < stop && in < a.inner && col < a.outer;
    float4 v[4] = {};
    if (there) {
#pragma unroll 2
      for (int b = first + turn; b <= last; b += lanes) {
        const float4* p = reinterpret_cast<const float4*>(sums(b)) + block * 4 * THREADS + thread;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float4 f = p[q * THREADS];
          v[q].x += f.x;
          v[q].y += f.y;
          v[q].z += f.z;
          v[q].w += f.w;
        }
      }
    }
    if (lanes > 1) {
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 4; ++q) meet[q][threadIdx.x] = v[q];
      __syncthreads();
      if (turn == 0) {
        for (int l = 1; l < lanes; ++l)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 f = meet[q][l * across + at];
            v[q].x += f.x;
            v[q].y += f.y;
            v[q].z += f.z;
            v[q].w += f.w;
          }
      }
    }
    if (turn == 0 && there) {
      const float r[16] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w,
                           v[2].x, v[2].y, v[2].z, v[2].w, v[3].x, v[3].y, v[3].z, v[3].w};
#pragma unroll
      for (int p = 0; p < 16 / N; ++p) {
        PieceV<T> out;
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = (T)r[p * N + i];
        const int c = col + p * N;
        T* to = dw + (int64_t)in * a.outer + c;
        if (c + N <= a.outer) *reinterpret_cast<typename Piece<T>::U*>(to) = out;
        else if (c < a.outer) store_first<T>(to, out, a.outer - c);
      }
    }
  }
  if (in0 == 0 && part == 0) {   // db
    float* one = reinterpret_cast<float*>(meet);
    for (int base = 0; base < BN; base += across) {
      const bool there = base + at < BN && col0 + base + at < a.outer;
      float v = 0.f;
      if (there) {
#pragma unroll 4
        for (int b = first + turn; b <= last; b += lanes) v += sums(b)[BR * BN + base + at];
      }
      __syncthreads();
      one[threadIdx.x] = v;
      __syncthreads();
      if (turn == 0 && there) {
        for (int l = 1; l < lanes; ++l) v += one[l * across + at];
        a.db[(int64_t)group * a.outer + col0 + base + at] = v;
      }
    }
  }
}

template <typename T, int BR, int BN>
int64_t weight_tiles(int inner, int outer) {
  return (int64_t)((inner + BR - 1) / BR) * ((outer + BN - 1) / BN);
}

template <typename T, int BR, int BN, int WR, int WN>
int launch_weights(ds_ctx* ctx, MmArgs& a, float* partial) {
  a.col_tiles = (a.outer + BN - 1) / BN;
  const int64_t tiles = weight_tiles<T, BR, BN>(a.inner, a.outer), chunks = ds_weight_chunks(a.rows, tiles, 128 / (int)sizeof(T));
  const int64_t wgs = (tiles * chunks + 7) / 8 * 8;
  if (wgs > ds_most_workgroups(64 * WR * WN)) return ds_fail(ctx, DS_EINVAL, "weights of %d by %d are more tiles than a launch has", a.inner, a.outer);
  const bool direct = sixteen(a.x, a.xs, sizeof(T)) && sixteen(a.dy, a.dys, sizeof(T)) && a.inner % Piece<T>::N == 0 && a.outer % Piece<T>::N == 0;
  const dim3 grid((unsigned)wgs), block(64 * WR * WN);
  if (direct) hipLaunchKernelGGL(HIP_KERNEL_NAME(weight_tiles_kernel<T, BR, BN, WR, WN, true>), grid, block, 0, ctx->stream, a, partial, (int)chunks);
  else hipLaunchKernelGGL(HIP_KERNEL_NAME(weight_tiles_kernel<T, BR, BN, WR, WN, false>), grid, block, 0, ctx->stream, a, partial, (int)chunks);
  // threads to a unit by the chunks that a group has on average; workgroups for about 2,048 in all
  const int64_t of_group = chunks / (a.groups < chunks ? a.groups : chunks) + 1;
  const int lanes = of_group > 16 ? 8 : of_group > 8 ? 4 : of_group > 4 ? 2 : 1;
  const int64_t units = (int64_t)(BR / WR / 32) * (BN / WN / 32) * 64 * WR * WN * lanes / kJoin;
  int64_t parts = 2048 / (tiles * a.groups);
  parts = parts < 1 ? 1 : parts < units ? parts : units;
  hipLaunchKernelGGL(HIP_KERNEL_NAME(weight_join_kernel<T, BR, BN, WR, WN>), dim3((unsigned)(tiles * parts), a.groups), dim3(kJoin), 0, ctx->stream, a,
                     partial, (int)chunks, (int)parts, lanes);
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

template <typename T, bool TRANSPOSED>
int launch_rows(ds_ctx* ctx, MmArgs& a) {
  if (ds_narrow_tiles(a.rows, a.groups, TRANSPOSED ? a.inner : a.outer) <= kNarrowTiles) return launch<T, 128, 128, 2, 2, TRANSPOSED>(ctx, a);
  return launch<T, 256, 256, 2, 4, TRANSPOSED>(ctx, a);
}

int ds_launch_row_tiles(ds_ctx* ctx, int dtype, bool transposed, MmArgs& a) {
  if (dtype == DS_ELEM_F32) {
    if (ds_wide_tiles(a.rows, transposed ? a.inner : a.outer)) return transposed ? launch<float, 256, 128, 4, 2, true>(ctx, a) : launch<float, 256, 128, 4, 2, false>(ctx, a);
    return transposed ? launch<float, 128, 128, 2, 4, true>(ctx, a) : launch<float, 128, 128, 2, 4, false>(ctx, a);
  }
  if (dtype == DS_ELEM_BF16) return transposed ? launch_rows<__bf16, true>(ctx, a) : launch_rows<__bf16, false>(ctx, a);
  return transposed ? launch_rows<_Float16, true>(ctx, a) : launch_rows<_Float16, false>(ctx, a);
}

int64_t ds_weight_tiles_bytes(int dtype, int rows, int inner, int outer) {
  const int64_t side = dtype == DS_ELEM_F32 ? 128 : 256;
  const int64_t tiles = dtype == DS_ELEM_F32 ? weight_tiles<float, 128, 128>(inner, outer) : weight_tiles<__bf16, 256, 256>(inner, outer);
  const int64_t chunks = ds_weight_chunks(rows, tiles, dtype == DS_ELEM_F32 ? 32 : 64);
  return chunks > 1 ? tiles * chunks * 2 * (side * side + side) * (int64_t)sizeof(float) : 0;
}

int ds_launch_weight_tiles(ds_ctx* ctx, int dtype, MmArgs& a, void* partial) {
  if (dtype == DS_ELEM_F32) return launch_weights<float, 128, 128, 2, 4>(ctx, a, (float*)partial);
  if (dtype == DS_ELEM_BF16) return launch_weights<__bf16, 256, 256, 2, 4>(ctx, a, (float*)partial);
  return launch_weights<_Float16, 256, 256, 2, 4>(ctx, a, (float*)partial);
}
