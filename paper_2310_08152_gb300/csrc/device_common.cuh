// Device helpers shared by the sm_103a kernels: 16-bit element types, the RoPE angle, and PTX
// wrappers for mbarriers, bulk copies, the global timer and programmatic dependent launch.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

namespace kvc {

// ---------------------------------------------------------------------------------------------
// 16-bit element types
// ---------------------------------------------------------------------------------------------
struct F16T {
  static __device__ __forceinline__ float2 f2(uint32_t u) {
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
  }
  static __device__ __forceinline__ float f1(uint16_t u) { return __half2float(__ushort_as_half(u)); }
  static __device__ __forceinline__ uint16_t r(float x) { return __half_as_ushort(__float2half_rn(x)); }
  static __device__ __forceinline__ uint32_t r2(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
struct BF16T {
  static __device__ __forceinline__ float2 f2(uint32_t u) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&u));
  }
  static __device__ __forceinline__ float f1(uint16_t u) { return __bfloat162float(__ushort_as_bfloat16(u)); }
  static __device__ __forceinline__ uint16_t r(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }
  static __device__ __forceinline__ uint32_t r2(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

// ---------------------------------------------------------------------------------------------
// RoPE angle.  theta = pos * base^(-2i/rot) is reduced in turns: g = base^(-2i/rot) / (2 pi) is
// held as a double-float (hi, lo); pos * hi is split exactly with an FMA (Dekker's two-product),
// the integer part of the turns is removed exactly, leaving f in [-1/2, 1/2] turns with an error
// near 1e-7 at any position below 2^24 (a plain binary32 product would be off by up to half an ulp
// of theta, about 5e-4 rad at position 8192).  The sine and cosine of 2 pi f, an angle in
// [-pi, pi], come from the hardware approximation, whose absolute error there (about 2^-21) is
// far below the 16-bit rounding of the rotated values (2^-11 relative for fp16).
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float rope_turns(int32_t pos, float2 g) {
  const float p = (float)pos;
  const float a = __fmul_rn(p, g.x);
  const float e = __fmaf_rn(p, g.x, -a);
  return __fadd_rn(__fsub_rn(a, rintf(a)), __fmaf_rn(p, g.y, e));
}
__device__ __forceinline__ void rope_sincos(int32_t pos, float2 g, float* s, float* c) {
  __sincosf(6.28318530717958647692f * rope_turns(pos, g), s, c);
}
// The same to the last bits of binary32, where the rotated query is not rounded to 16 bits and the outputs are held to
// more than that: the approximation's 2^-21 was half of the output's error (1.4e-6 against 64 bits, 8 samples of a prefix
// of 800 rows).
__device__ __forceinline__ void rope_sincos_full(int32_t pos, float2 g, float* s, float* c) {
  sincospif(2.f * rope_turns(pos, g), s, c);
}

// Two 32-bit values as a sum of packed 16-bit parts: the first rounds them, each later one rounds what is left, which
// binary32 holds exactly.  Two parts of f16 hold 22 bits of a value, three of bf16 all 24.
template <typename T>
constexpr int kFullParts = 2;
template <>
constexpr int kFullParts<BF16T> = 3;
// With LARGE the first part ends at f16's largest value, so that the sum reaches twice that: two turned columns may be
// sqrt(2) times the larger of them.  (What is past 65,504 has 11 bits, in steps of 16, where the query's own are of 32.)
template <typename T, int N, bool LARGE = false>
__device__ __forceinline__ void split_parts(float x, float y, uint32_t* part) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (LARGE && std::is_same_v<T, F16T>)
      part[i] = i == 0 ? T::r2(fminf(fmaxf(x, -65504.f), 65504.f), fminf(fmaxf(y, -65504.f), 65504.f)) : T::r2(x, y);
    else
      part[i] = T::r2(x, y);
    if (i + 1 < N) {
      const float2 back = T::f2(part[i]);
      x -= back.x;
      y -= back.y;
    }
  }
}

// Chunk c (eight columns) of a query as packed 16-bit parts, rotated at pos where NQ > 1 (the first `rot` columns; rot is a
// multiple of 16).  q is 16-byte aligned.
template <typename T, int NQ>
__device__ __forceinline__ void query_chunk(const uint16_t* q, int c, int rot, int32_t pos, const float2* rope_g,
                                            uint32_t (&part)[NQ][4]) {
  const uint4 x = *reinterpret_cast<const uint4*>(q + c * 8);
  const uint32_t a[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) part[0][e] = a[e];
#pragma unroll
  for (int i = 1; i < NQ; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[i][e] = 0;
  if (NQ == 1 || c * 8 >= rot) return;
  const int half = rot / 2;
  const bool first = c * 8 < half;
  const int i0 = first ? c * 8 : c * 8 - half;
  const uint4 y = *reinterpret_cast<const uint4*>(q + (first ? c * 8 + half : i0));
  const uint32_t b[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 u = T::f2(a[e]), v = T::f2(b[e]);
    float sn0, cs0, sn1, cs1;
    rope_sincos_full(pos, rope_g[i0 + 2 * e], &sn0, &cs0);
    rope_sincos_full(pos, rope_g[i0 + 2 * e + 1], &sn1, &cs1);
    uint32_t out[NQ];
    split_parts<T, NQ, true>(first ? u.x * cs0 - v.x * sn0 : u.x * cs0 + v.x * sn0,
                             first ? u.y * cs1 - v.y * sn1 : u.y * cs1 + v.y * sn1, out);
#pragma unroll
    for (int i = 0; i < NQ; ++i) part[i][e] = out[i];
  }
}

// ---------------------------------------------------------------------------------------------
// PTX helpers: mbarrier, 1-D bulk copy (TMA), global timer
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void fence_mbar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ uint64_t global_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
// Waits for the phase with the given parity; gives up after limit_ns (returns false).
__device__ __forceinline__ bool mbar_wait_bounded(uint64_t* bar, uint32_t parity, unsigned long long limit_ns) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_ns();
  for (uint32_t it = 1;; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 0 && global_ns() - t0 > limit_ns) return false;
  }
}
// Programmatic dependent launch: let the next kernel on the stream be scheduled, and wait for
// the preceding one (no-ops when the launch did not opt in).
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void bulk_g2s(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_addr(dst)),
               "l"(src), "r"(bytes), "r"(smem_addr(bar))
               : "memory");
}
// Orders this thread's generic-proxy shared-memory writes before later async-proxy accesses
// (bulk copies, tensor-core operand reads).
__device__ __forceinline__ void fence_proxy_async_smem() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

}  // namespace kvc
