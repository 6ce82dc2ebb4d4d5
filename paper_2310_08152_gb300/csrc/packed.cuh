// Rows of 4 bits, shared by the kernels that write and read them (packed.cu, copy.cu).
//
// The columns of a row are in groups of 32 (the last one of 16 where D is 80).  A group has its least value lo and a step,
// both in the cache's 16-bit type: the step is a fifteenth of the group's range, rounded up to that type (0 below 2^-126,
// where its reciprocal would not be finite).  Column x has the code rint((x - lo) / step), from 0 to 15, with the product
// by 1 / step in binary32, and stands for lo + step * code.  Rounding the step up keeps the group's largest value within
// half a step of code 15; a group that holds a NaN or an infinity has a step of NaN and reads as NaN.
//
// A row's codes are D / 8 words, word w the columns 8 w .. 8 w + 7 from its low bits up; its (lo, step) pairs are a word a
// group, the step in the high half.  Codes and pairs are planes of their own, in the layout of the rows.
#pragma once

#include "device_common.cuh"

namespace kvc {

// (lo, step) of a pair.
__device__ __forceinline__ float2 pair_values(uint32_t pair, F16T) { return F16T::f2(pair); }
__device__ __forceinline__ float2 pair_values(uint32_t pair, BF16T) {
  return make_float2(__uint_as_float(pair << 16), __uint_as_float(pair & 0xFFFF0000u));
}

template <int D>
struct PackedRow {
  static constexpr int G = (D + 31) / 32;  // groups
  static constexpr int W = D / 8;          // code words
  static constexpr int CP = 4 * G;         // lanes a row: one for 8 columns, four for a group (two of them idle at D 80)
  static constexpr int RB = D / 2;         // bytes of codes
  static constexpr int PB = 4 * G;         // bytes of pairs
};

__device__ __forceinline__ uint16_t round_up16(float x, F16T) { return __half_as_ushort(__float2half_ru(x)); }
__device__ __forceinline__ uint16_t round_up16(float x, BF16T) { return __bfloat16_as_ushort(__float2bfloat16_ru(x)); }

// The code word of a lane's eight columns (values of the 16-bit type T), and the (lo, step) pair of its group, whose four
// lanes are consecutive and call this together.  A lane without columns is not `active`.
template <typename T>
__device__ __forceinline__ uint32_t pack8(const float (&x)[8], bool active, uint32_t* pair) {
  float lo = x[0], hi = x[0], odd = x[0] * 0.f;  // odd: NaN if a value is not finite
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
    odd = fmaf(x[e], 0.f, odd);
  }
  if (!active) {
    lo = INFINITY;
    hi = -INFINITY;
    odd = 0.f;
  }
#pragma unroll
  for (int i = 1; i <= 2; i <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, i));
    hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, i));
    odd += __shfl_xor_sync(0xFFFFFFFFu, odd, i);
  }
  float s = __fdiv_rn(__fsub_rn(hi, lo) + odd, 15.f);
  if (s < 1.17549435e-38f) s = 0.f;
  const uint16_t s16 = round_up16(s, T{});
  const float step = T::f1(s16);
  const float inv = step > 0.f ? __frcp_rn(step) : 0.f;
  uint32_t word = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // adding 2^23 leaves the nearest whole number (ties to even) in the low bits
    const float t = fminf(__fmul_rn(__fsub_rn(x[e], lo), inv), 15.f);
    word |= (__float_as_uint(__fadd_rn(t, 8388608.f)) & 15u) << (4 * e);
  }
  *pair = (uint32_t)T::r(lo) | (uint32_t)s16 << 16;
  return word;
}

}  // namespace kvc
