// Rows of 4 bits, shared by the kernels that write and read them (packed.cu, copy.cu).
//
// The columns of a row are in groups of 32 (the last one of 16 where D is 80).  A group has its least value lo and a step,
// both in the cache's 16-bit type: the step is a fifteenth of the group's range, rounded up to that type (0 below 2^-126,
// where its reciprocal would not be finite).  Column x has the code rint((x - lo) / step), from 0 to 15, with the product
// by 1 / step in binary32, and stands for lo + step * code.  Rounding the step up keeps the group's largest value within
// half a step of code 15; a group that holds a NaN or an infinity has a step and a least value of NaN.
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

// The smaller and the greater of packed values; NaN where one is.
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b, F16T) {
  const __half2 r = __hmin2_nan(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b, BF16T) {
  const __nv_bfloat162 r = __hmin2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, F16T) {
  const __half2 r = __hmax2_nan(*reinterpret_cast<__half2*>(&a), *reinterpret_cast<__half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b, BF16T) {
  const __nv_bfloat162 r = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// The least and, negated, the greatest of n words of packed values.
template <typename T>
__device__ __forceinline__ uint32_t range_of(const uint32_t* w, int n) {
  uint32_t lo = w[0], hi = w[0];
#pragma unroll
  for (int i = 1; i < n; ++i) {
    lo = min2(lo, w[i], T{});
    hi = max2(hi, w[i], T{});
  }
  lo = min2(lo, __byte_perm(lo, lo, 0x1032), T{});
  hi = max2(hi, __byte_perm(hi, hi, 0x1032), T{});
  return __byte_perm(lo, hi, 0x5410) ^ 0x80000000u;
}

// A group's (lo, step) pair from its range, lo, and 1 / step (0 where the step is 0).
template <typename T>
__device__ __forceinline__ uint32_t group_pair(uint32_t range, float* lo, float* inv) {
  uint32_t lo16 = range & 0xFFFFu;
  *lo = T::f1((uint16_t)lo16);
  float s = __fdiv_rn(__fsub_rn(T::f1((uint16_t)(range >> 16 ^ 0x8000u)), *lo), 15.f);
  s = fmaf(s, 0.f, s);  // NaN where it is not finite
  if (s != s) lo16 = 0x7FFFu;
  if (s < 1.17549435e-38f) s = 0.f;
  const uint32_t s16 = round_up16(s, T{});
  const float step = T::f1((uint16_t)s16);
  *inv = step > 0.f ? __frcp_rn(step) : 0.f;
  return lo16 | s16 << 16;
}

// x - y for a 16-bit x, in one instruction.
__device__ __forceinline__ float sub_mixed(uint32_t x, float y, F16T) {
  float d;
  asm("sub.f32.f16 %0, %1, %2;" : "=f"(d) : "h"((uint16_t)x), "f"(y));
  return d;
}
__device__ __forceinline__ float sub_mixed(uint32_t x, float y, BF16T) {
  float d;
  asm("sub.f32.bf16 %0, %1, %2;" : "=f"(d) : "h"((uint16_t)x), "f"(y));
  return d;
}

// The code word of eight columns.  Adding 2^23 leaves the nearest whole number (ties to even) in the low bits of the sum;
// the word is those bits in base 16, where the upper ones come to a constant.  A column is four instructions of the FMA pipe.
// (With masks, shifts and a clamp for each, and a step and its reciprocal for every eight columns, 8,000 rows of 80 columns
// in 8 layers of 32 heads went to 4 bits in 494 us instead of 133.)
template <typename T>
__device__ __forceinline__ uint32_t code_word(const uint32_t* w, float lo, float inv) {
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    b[e] = __float_as_uint(__fadd_rn(__fmul_rn(sub_mixed(w[e / 2] >> (16 * (e & 1)), lo, T{}), inv), 8388608.f));
  uint32_t y = b[7];
#pragma unroll
  for (int e = 6; e >= 0; --e) y = y * 16u + b[e];
  return y - (0x4B000000u + 0xB0000000u);
}

// A lane's group gi of a row of 16-bit values (16-byte aligned): its pair and its code words, of which a group of 16 columns
// has two.
template <typename T, int D>
__device__ __forceinline__ uint32_t pack_group(const uint16_t* row, int gi, uint32_t (&code)[4]) {
  const uint4* from = reinterpret_cast<const uint4*>(row + 32 * gi);
  const bool whole = D % 32 == 0 || gi + 1 < PackedRow<D>::G;
  uint32_t x[16];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint4 v = e < 2 || whole ? __ldg(from + e) : make_uint4(0, 0, 0, 0);
    x[4 * e] = v.x, x[4 * e + 1] = v.y, x[4 * e + 2] = v.z, x[4 * e + 3] = v.w;
  }
  if (!whole) {
#pragma unroll
    for (int e = 8; e < 16; ++e) x[e] = x[e - 8];
  }
  float lo, inv;
  const uint32_t pair = group_pair<T>(range_of<T>(x, 16), &lo, &inv);
#pragma unroll
  for (int e = 0; e < 4; ++e) code[e] = code_word<T>(x + 4 * e, lo, inv);
  return pair;
}

// Stores it as group gi of row `row` of the planes.
template <int D>
__device__ __forceinline__ void store_group(unsigned char* codes, uint32_t* pairs, int64_t row, int gi,
                                            const uint32_t (&code)[4], uint32_t pair) {
  using R = PackedRow<D>;
  uint32_t* to = reinterpret_cast<uint32_t*>(codes) + row * R::W + 4 * gi;
  if constexpr (D % 32 == 0) {
    *reinterpret_cast<uint4*>(to) = make_uint4(code[0], code[1], code[2], code[3]);
  } else {  // rows of 40 bytes
    *reinterpret_cast<uint2*>(to) = make_uint2(code[0], code[1]);
    if (gi + 1 < R::G) *reinterpret_cast<uint2*>(to + 2) = make_uint2(code[2], code[3]);
  }
  pairs[row * R::G + gi] = pair;
}

// Of a lane's eight columns: the code word, and the pair of the group, whose four lanes are consecutive and call this
// together.  A lane without columns is not `active`.
template <typename T>
__device__ __forceinline__ uint32_t pack8(const uint32_t (&w)[4], bool active, uint32_t* pair) {
  constexpr uint32_t kInf = std::is_same_v<T, F16T> ? 0x7C007C00u : 0x7F807F80u;  // least, and negated greatest
  uint32_t r = active ? range_of<T>(w, 4) : kInf;
  r = min2(r, __shfl_xor_sync(0xFFFFFFFFu, r, 1), T{});
  r = min2(r, __shfl_xor_sync(0xFFFFFFFFu, r, 2), T{});
  float lo, inv;
  *pair = group_pair<T>(r, &lo, &inv);
  return code_word<T>(w, lo, inv);
}

// A column pair of a code word, its codes c and c' at bits 4 e and 4 e + 16, as the values that they stand for.
__device__ __forceinline__ float2 code_values(uint32_t w, int e, float2 pair) {
  const uint32_t x = (w >> (4 * e) & 0x000F000Fu) | 0x64006400u;  // 1024 + c
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half(0x6400)));
  const float2 c = __half22float2(h);
  return make_float2(fmaf(pair.y, c.x, pair.x), fmaf(pair.y, c.y, pair.x));
}

}  // namespace kvc
