// Rows held in 8 bits: what a code and a scale stand for, on the GPU.
//
// A code is an e4m3 number (sign, 4 bits of exponent, 3 of fraction; 448 is the largest, 2^-9 the smallest, no infinities), and 32 neighbouring columns of a row
// share a power of two, of which the exponent is kept: x ~ code * 2^(scale - 127).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "rows.h"

namespace {

#define DS_GLOBAL __attribute__((address_space(1)))

constexpr int kPackBlock = 32;   // columns that share a scale

// 2^(s - 127)
__device__ __forceinline__ float power_of_scale(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x400000u); }

// N codes, each in a byte of its own
template <int N>
using PackedPiece = typename std::conditional<N == 8, uint64_t, typename std::conditional<N == 4, uint32_t, typename std::conditional<N == 2, uint16_t, uint8_t>::type>::type>::type;
template <int N>
__device__ __forceinline__ PackedPiece<N> load_codes(const uint8_t* p) {
  typedef PackedPiece<N> U __attribute__((aligned(1)));
  return *reinterpret_cast<const U*>(p);
}
// without the first `by` (at most N), zeros behind the others
template <int N>
__device__ __forceinline__ PackedPiece<N> shifted_codes(PackedPiece<N> v, unsigned by) {
  return by >= N ? 0 : (PackedPiece<N>)(v >> (8 * by));
}
// the first `have` of N from p on, zeros behind them; nothing outside of them is read
template <int N>
__device__ __forceinline__ PackedPiece<N> load_first_codes(const uint8_t* p, int have) {
  if (have >= N) return load_codes<N>(p);
  PackedPiece<N> v = 0;
#pragma unroll
  for (int i = 0; i < N - 1; ++i)
    if (i < have) v |= (PackedPiece<N>)((PackedPiece<N>)p[i] << (8 * i));
  return v;
}

// The four codes of a word times their power of two. (The instruction takes the power from the bits of an fp32 number's exponent.)
__device__ __forceinline__ void four_of(uint32_t word, float power, __bf16 (&to)[4]) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, power, true);
  to[0] = lo[0];
  to[1] = lo[1];
  to[2] = hi[0];
  to[3] = hi[1];
}
__device__ __forceinline__ void four_of(uint32_t word, float power, _Float16 (&to)[4]) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, power, true);
  to[0] = lo[0];
  to[1] = lo[1];
  to[2] = hi[0];
  to[3] = hi[1];
}
__device__ __forceinline__ void four_of(uint32_t word, float power, float (&to)[4]) {
  const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, power, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(word, power, true);
  to[0] = lo[0];
  to[1] = lo[1];
  to[2] = hi[0];
  to[3] = hi[1];
}
// What a piece of codes stands for
template <typename T>
__device__ __forceinline__ typename Piece<T>::V decoded(PackedPiece<Piece<T>::N> codes, uint32_t scale) {
  constexpr int N = Piece<T>::N;
  const float power = __uint_as_float(scale << 23);
  typename Piece<T>::V v;
#pragma unroll
  for (int q = 0; q < N / 4; ++q) {
    T four[4];
    four_of((uint32_t)((uint64_t)codes >> (32 * q)), power, four);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * q + i] = four[i];
  }
  return v;
}

// A gate of dx: open where its value is above 0 (an infinity's code is that of a NaN, which is not). `load` is a piece, zeros behind the matrix' end; `at` one as it
// stands, and `behind` what is left of it where it was read `by` elements in front of its place: nothing waits for a load where it is asked for.
template <typename T, bool PACKED>
struct RowGate {
  typedef T E;
  typedef typename Piece<T>::V V;
  static __device__ __forceinline__ V load(const T* p, const T* end) { return load_within<T>(p, end); }
  static __device__ __forceinline__ V at(const T* p) { return *(const DS_GLOBAL typename Piece<T>::U*)p; }
  static __device__ __forceinline__ V behind(V v, unsigned by) { return shifted<T>(v, by); }
  static __device__ __forceinline__ V load_first(const T* p, int have) { return load_piece<T>(p, have); }
  static __device__ __forceinline__ bool is_open(V v, int i) { return (float)v[i] > 0.f; }
  static __device__ __forceinline__ PieceV<T> through(V gate, PieceV<T> v) {
#pragma unroll
    for (int i = 0; i < Piece<T>::N; ++i) v[i] = is_open(gate, i) ? v[i] : (T)0.f;
    return v;
  }
};
template <typename T>
struct RowGate<T, true> {
  static constexpr int N = Piece<T>::N;
  typedef uint8_t E;
  typedef PackedPiece<N> V;
  static __device__ __forceinline__ V load(const uint8_t* p, const uint8_t* end) {   // (a matrix has N bytes)
    const int64_t by = p + N - end;
    const V v = load_codes<N>(by <= 0 ? p : end - N);
    return by <= 0 ? v : shifted_codes<N>(v, by < N ? (unsigned)by : N);
  }
  static __device__ __forceinline__ V at(const uint8_t* p) {
    typedef V U __attribute__((aligned(1)));
    return *(const DS_GLOBAL U*)p;
  }
  static __device__ __forceinline__ V behind(V v, unsigned by) { return shifted_codes<N>(v, by); }
  static __device__ __forceinline__ V load_first(const uint8_t* p, int have) { return load_first_codes<N>(p, have); }
  static __device__ __forceinline__ bool is_open(V v, int i) { return (uint32_t)((v >> (8 * i)) & 255) - 1u < 126u; }
  // (four codes at a time: a byte's highest bit says that it is 1 to 126, and then is all of its bits)
  static __device__ __forceinline__ PieceV<T> through(V gate, PieceV<T> v) {
    union {
      PieceV<T> piece;
      uint32_t word[4];
    } u;
    u.piece = v;
#pragma unroll
    for (int q = 0; q < N / 4; ++q) {
      const uint32_t c = (uint32_t)((uint64_t)gate >> (32 * q)), low = c & 0x7f7f7f7fu;
      const uint32_t high = (low + 0x7f7f7f7fu) & ~((low + 0x01010101u) | c) & 0x80808080u, whole = high | (high - (high >> 7));
      if constexpr (sizeof(T) == 2) {
        u.word[2 * q] &= __builtin_amdgcn_perm(whole, whole, 0x01010000u);
        u.word[2 * q + 1] &= __builtin_amdgcn_perm(whole, whole, 0x03030202u);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) u.word[4 * q + i] &= (uint32_t)((int32_t)(whole << (24 - 8 * i)) >> 31);
      }
    }
    return u.piece;
  }
};

}  // namespace
