// Rows held in 8 bits: what a code and a scale stand for, on the GPU.
//
// A code is an e4m3 number (sign, 4 bits of exponent, 3 of fraction; 448 is the largest, 2^-9 the smallest, no infinities), and 32 neighbouring columns of a row
// share a power of two, of which the exponent is kept: x ~ code * 2^(scale - 127).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

constexpr int kPackBlock = 32;   // columns that share a scale

// 2^(s - 127)
__device__ __forceinline__ float power_of_scale(uint32_t s) { return __uint_as_float(s ? s << 23 : 0x400000u); }

}  // namespace
