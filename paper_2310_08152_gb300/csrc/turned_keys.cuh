// The rotation of keys, shared by the appends (kernels.cu, packed.cu).
#pragma once

#include <cuda_runtime.h>

namespace kvc {

// A key's columns x1 and x2, half a rotation apart, turned by (cos, sin) of their angle.  Each product and sum is spelled out,
// as a compiler that fuses either product with the sum would round the keys of one kernel unlike another's: the same tokens have
// to give the same rows in every append, and the same codes from an append to 4 bits as from a copy of the 16-bit rows.
__device__ __forceinline__ float turned_first(float x1, float x2, float2 cs) { return __fmaf_rn(x1, cs.x, -__fmul_rn(x2, cs.y)); }
__device__ __forceinline__ float turned_second(float x1, float x2, float2 cs) { return __fmaf_rn(x1, cs.y, __fmul_rn(x2, cs.x)); }

}  // namespace kvc
