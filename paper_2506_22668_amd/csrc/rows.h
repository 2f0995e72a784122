// What the operators on rows of features share: 16-byte pieces of a row at any alignment, sums over the lanes of a row, and the
// rows of a group.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "group_range.h"

namespace {

// 16 bytes of a row. `U` is only as aligned as an element: rows of any width, stride and start are read and written in
// 16-byte accesses (the GPU runs with unaligned access enabled), so that no second form for odd rows is needed.
template <typename T>
struct Piece;
template <>
struct Piece<float> {
  static constexpr int N = 4;
  typedef float V __attribute__((ext_vector_type(4)));
  typedef float U __attribute__((ext_vector_type(4), aligned(4)));
};
template <>
struct Piece<__bf16> {
  static constexpr int N = 8;
  typedef __bf16 V __attribute__((ext_vector_type(8)));
  typedef __bf16 U __attribute__((ext_vector_type(8), aligned(2)));
};
template <>
struct Piece<_Float16> {
  static constexpr int N = 8;
  typedef _Float16 V __attribute__((ext_vector_type(8)));
  typedef _Float16 U __attribute__((ext_vector_type(8), aligned(2)));
};

// the first `have` elements from p on, zeros behind them; nothing outside of them is read
template <typename T>
__device__ __forceinline__ typename Piece<T>::V load_piece(const T* p, int have) {
  if (have >= Piece<T>::N) return *reinterpret_cast<const typename Piece<T>::U*>(p);
  typename Piece<T>::V v = {};
#pragma unroll
  for (int i = 0; i < Piece<T>::N - 1; ++i)
    if (i < have) v[i] = p[i];
  return v;
}

template <typename T>
using PieceV = typename Piece<T>::V;

// without the first `by` (at most N) elements, zeros behind the others
template <typename T>
__device__ __forceinline__ PieceV<T> shifted(PieceV<T> v, unsigned by) {
  union {
    PieceV<T> piece;
    unsigned __int128 bits;
  } u;
  u.piece = v;
  u.bits = by >= Piece<T>::N ? 0 : u.bits >> (8 * (int)sizeof(T) * by);
  return u.piece;
}

// 16 bytes from p on; behind `end`, where the matrix ends, zeros, and nothing is read there. (A matrix has 16 bytes.)
template <typename T>
__device__ __forceinline__ PieceV<T> load_within(const T* p, const T* end) {
  constexpr int N = Piece<T>::N;
  const int64_t by = p + N - end;
  const PieceV<T> v = *reinterpret_cast<const typename Piece<T>::U*>(by <= 0 ? p : end - N);
  return by <= 0 ? v : shifted<T>(v, by < N ? (unsigned)by : N);
}

template <typename T>
__device__ __forceinline__ PieceV<T> first_elements(PieceV<T> v, int have) {
#pragma unroll
  for (int i = 0; i < Piece<T>::N; ++i) v[i] = i < have ? v[i] : (T)0.f;
  return v;
}

// the first `have` (1 to N - 1) elements
template <typename T>
__device__ __forceinline__ void store_first(T* p, PieceV<T> v, int have) {
  constexpr int N = Piece<T>::N;
  typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  typedef T Two __attribute__((ext_vector_type(2), aligned(sizeof(T))));
  if constexpr (N == 8) {
    if (have & 4) {
      *reinterpret_cast<Four*>(p) = Four{v[0], v[1], v[2], v[3]};
      p += 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = v[i + 4];
    }
  }
  if (have & 2) {
    *reinterpret_cast<Two*>(p) = Two{v[0], v[1]};
    p += 2;
    v[0] = v[2];
  }
  if (have & 1) *p = v[0];
}

template <typename T>
__device__ __forceinline__ void store_piece(T* p, PieceV<T> v, int have) {
  if (have >= Piece<T>::N) *reinterpret_cast<typename Piece<T>::U*>(p) = v;
  else if (have > 0) store_first<T>(p, v, have);
}

// N neighbouring elements of a row
template <typename T, int N>
struct Elements {
  typedef T V __attribute__((ext_vector_type(N)));
  typedef T U __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Those from `col` (< cols) on; of rows of N or more, where fewer are left, the row's last N, which settle moves to their place (TINY: rows of fewer, one by one)
template <typename T, int N, bool TINY>
__device__ __forceinline__ typename Elements<T, N>::V load_elements(const T* row, int col, int cols) {
  if constexpr (TINY) {
    typename Elements<T, N>::V v = {};
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (col + i < cols) v[i] = row[col + i];
    return v;
  } else {
    return *reinterpret_cast<const typename Elements<T, N>::U*>(row + min(col, cols - N));
  }
}
template <typename T, int N, bool TINY>
__device__ __forceinline__ void settle_elements(typename Elements<T, N>::V& v, int col, int cols) {
  if constexpr (!TINY) {
    const int by = col + N - cols;
    if (by <= 0) return;
#pragma unroll
    for (int s = 1; s < N; ++s)
      if (by >= s) {
#pragma unroll
        for (int i = 0; i + 1 < N; ++i) v[i] = v[i + 1];
      }
  }
}

template <int CTRL>
__device__ __forceinline__ float add_across(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over groups of LANES neighbouring lanes, in every lane of the group: exchanges inside the registers, no LDS.
template <int LANES>
__device__ __forceinline__ float sum_lanes(float v) {
  if constexpr (LANES >= 2) v = add_across<0xB1>(v);    // lane ^ 1
  if constexpr (LANES >= 4) v = add_across<0x4E>(v);    // lane ^ 2
  if constexpr (LANES >= 8) v = add_across<0x141>(v);   // 7 - lane: the other four
  if constexpr (LANES >= 16) v = add_across<0x140>(v);  // 15 - lane: the other eight
  if constexpr (LANES >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  if constexpr (LANES >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  return v;
}

struct GroupTile {
  int group;            // == groups: rows of no group
  int begin, end;       // positions in the order
};

// The rows cut into tiles of 2^shift, group by group, the rows of no group last. Used by whole waves, with the same answer in
// every lane: a lane holds one of 64 neighbouring groups, so that up to 64 groups are looked at once and a tile is found by a ballot.
class GroupTiles {
 public:
  __device__ __forceinline__ GroupTiles(const int64_t* offsets, int groups, int rows, int shift)
      : offsets_(offsets), groups_(groups), rows_(rows), shift_(shift) {
    look(0, 0);
  }
  // number of tiles
  __device__ __forceinline__ int count() {
    while (base_ + 64 <= groups_) look(base_ + 64, last_);
    return last_;
  }
  // tile 0 .. count() - 1
  __device__ __forceinline__ GroupTile find(int tile) {
    if (tile < before_) look(0, 0);
    while (tile >= last_ && base_ + 64 <= groups_) look(base_ + 64, last_);
    const unsigned long long reach = __ballot(upto_ > tile);
    const int src = reach ? __ffsll((long long)reach) - 1 : 63;
    const int g = __builtin_amdgcn_readfirstlane(src);
    const int first = __builtin_amdgcn_readlane(upto_ - tiles_, g);   // (where the sum is capped, before its first tile: the tile lies in its rows all the same)
    const int b = __builtin_amdgcn_readlane(begin_, g), e = __builtin_amdgcn_readlane(end_, g);
    GroupTile t;
    t.group = base_ + g;
    t.begin = b + ((tile - first) << shift_);
    t.end = min(e, t.begin + (1 << shift_));
    return t;
  }

 private:
  const int64_t* offsets_;
  int groups_, rows_, shift_;
  int base_, before_, last_;           // the first of the 64 groups; tiles in front of them and up to their end
  int begin_, end_, tiles_, upto_;     // of the lane's group
  __device__ __forceinline__ void look(int base, int before) {
    const int lane = threadIdx.x & 63, g = base + lane;
    base_ = base;
    before_ = before;
    begin_ = end_ = 0;
    if (g <= groups_) ds_group_range(offsets_, groups_, rows_, g, &begin_, &end_);
    tiles_ = ds_parts_of(begin_, end_, 1 << shift_);
    upto_ = tiles_;
    const int most = ds_most_parts(rows_, 1 << shift_, groups_ + 1);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(upto_, o, 64);
      if (lane >= o) upto_ = ds_add_parts(upto_, up, most);
    }
    upto_ = ds_add_parts(upto_, before, most);
    last_ = __builtin_amdgcn_readlane(upto_, 63);
  }
};

}  // namespace
