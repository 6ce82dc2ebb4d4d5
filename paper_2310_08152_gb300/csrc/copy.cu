// Sequences copied within a cache or from one to another, between 16 and 4 bits where the caches differ in that, and the
// scores of rows that are dropped.
//
// Every row of a source is read once, whatever the number of its targets: a block takes a run of rows of one (source, layer,
// K/V, head) stream into registers and stores it to each target.  What bounds a copy is memory: the bytes of the source once
// and of every target (8 samples of 4 prompts of up to 800 rows, 24 layers of 32 heads of 64: 725 us, 6.7 TB/s; between 16 and
// 4 bits 6.3 to 7.0 TB/s).
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernels.hpp"
#include "packed.cuh"

namespace kvc {
namespace {

constexpr int kCopyThreads = 256;
template <int DB>
constexpr int kCopyRows = copy_rows(DB);

// The device's view of a call's upload: in a kernel parameter or in the workspace.
struct CopyPlan {
  const CopySource* sources;
  const CopyTarget* targets;
};

struct CopyDev {
  Geometry g;
  CopySide src, dst;
  int n_chunks, n_sources;
};

__device__ __forceinline__ int64_t stream_row0(const Geometry& g, const CopySide& c, int m, int h, int s) {
  return (int64_t)m * g.H * c.C + c.st.seq_row0[s] + (int64_t)h * c.st.cap[s];
}

// Two values rounded to 16 bits, to the type's largest one where they are past it: a step that was rounded up may take a group's
// greatest value there.  A NaN stays one.
__device__ __forceinline__ uint32_t finite2(float lo, float hi, F16T) {
  uint32_t y;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}
__device__ __forceinline__ uint32_t finite2(float lo, float hi, BF16T) {
  uint32_t y;
  asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}

template <typename T, int D, int SB, int DB>
__device__ __forceinline__ void copy_block(const CopyDev& p, const CopyPlan& plan) {
  using R = PackedRow<D>;
  constexpr int CR = kCopyRows<DB>;
  const int chunk = blockIdx.x % p.n_chunks, sidx = blockIdx.x / p.n_chunks;
  int si = 0;  // the last source that begins at the chunk or before it; one without rows has none
  for (int z = p.n_sources; z - si > 1;) {
    const int mid = (si + z) / 2;
    if (plan.sources[mid].chunk0 <= chunk)
      si = mid;
    else
      z = mid;
  }
  const CopySource cs = plan.sources[si];
  const int r0 = (chunk - cs.chunk0) * CR;
  const int n = min(CR, cs.len - r0);
  const int h = sidx % p.g.H, kv = (sidx / p.g.H) & 1, m = sidx / (2 * p.g.H);
  const int tid = threadIdx.x;
  const int64_t row = stream_row0(p.g, p.src, m, h, cs.s) + r0;
  auto target_row = [&](int j) { return stream_row0(p.g, p.dst, m, h, plan.targets[cs.first + j].s) + r0; };

  if constexpr (SB == 16 && DB == 16) {
    constexpr int V = D / 8, U = CR * V / kCopyThreads;  // 16-byte vectors
    static_assert(CR * V % kCopyThreads == 0);
    const uint4* src = reinterpret_cast<const uint4*>((kv ? p.src.v : p.src.k) + row * D);
    uint4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (tid + u * kCopyThreads < n * V) x[u] = __ldcs(src + tid + u * kCopyThreads);
    for (int j = 0; j < cs.n; ++j) {
      uint4* dst = reinterpret_cast<uint4*>((kv ? p.dst.v : p.dst.k) + target_row(j) * D);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (tid + u * kCopyThreads < n * V) __stcs(dst + tid + u * kCopyThreads, x[u]);
    }
  } else if constexpr (SB == 4 && DB == 4) {
    constexpr int V = R::RB / 8, U = CR * V / kCopyThreads, UP = CR * R::G / kCopyThreads;  // 8-byte parts, pairs
    static_assert(CR * V % kCopyThreads == 0 && CR * R::G % kCopyThreads == 0);
    const uint2* src = reinterpret_cast<const uint2*>(kv ? p.src.pb.vc : p.src.pb.kc) + row * V;
    const uint32_t* sp = (kv ? p.src.pb.vp : p.src.pb.kp) + row * R::G;
    uint2 x[U];
    uint32_t y[UP];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (tid + u * kCopyThreads < n * V) x[u] = src[tid + u * kCopyThreads];
#pragma unroll
    for (int u = 0; u < UP; ++u)
      if (tid + u * kCopyThreads < n * R::G) y[u] = sp[tid + u * kCopyThreads];
    for (int j = 0; j < cs.n; ++j) {
      const int64_t to = target_row(j);
      uint2* dst = reinterpret_cast<uint2*>(kv ? p.dst.pb.vc : p.dst.pb.kc) + to * V;
      uint32_t* dp = (kv ? p.dst.pb.vp : p.dst.pb.kp) + to * R::G;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (tid + u * kCopyThreads < n * V) dst[tid + u * kCopyThreads] = x[u];
#pragma unroll
      for (int u = 0; u < UP; ++u)
        if (tid + u * kCopyThreads < n * R::G) dp[tid + u * kCopyThreads] = y[u];
    }
  } else if constexpr (SB == 16) {
    // a lane has a group: the range, the step and its reciprocal once, and four words of codes side by side
    constexpr int U = CR * R::G / kCopyThreads;
    static_assert(CR * R::G % kCopyThreads == 0);
    const uint16_t* src = (kv ? p.src.v : p.src.k) + row * D;
    const int64_t row_first = target_row(0);
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
      const int i = tid + u * kCopyThreads, r = i / R::G, gi = i % R::G;
      if (r >= n) break;
      uint32_t code[4];
      const uint32_t pair = pack_group<T, D>(src + r * D, gi, code);
      for (int j = 0; j < cs.n; ++j)
        store_group<D>(kv ? p.dst.pb.vc : p.dst.pb.kc, kv ? p.dst.pb.vp : p.dst.pb.kp,
                       (j == 0 ? row_first : target_row(j)) + r, gi, code, pair);
    }
  } else {
    // a lane has eight columns
    constexpr int U = CR * R::W / kCopyThreads;
    static_assert(CR * R::W % kCopyThreads == 0);
    const uint32_t* src = reinterpret_cast<const uint32_t*>(kv ? p.src.pb.vc : p.src.pb.kc) + row * R::W;
    const uint32_t* sp = (kv ? p.src.pb.vp : p.src.pb.kp) + row * R::G;
    uint32_t x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = tid + u * kCopyThreads;
      x[u] = y[u] = 0;
      if (i < n * R::W) {
        x[u] = __ldcs(src + i);
        y[u] = __ldg(sp + i / R::W * R::G + i % R::W / 4);
      }
    }
    uint4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float2 pv = pair_values(y[u], T{});
      const float2 a = code_values(x[u], 0, pv), b = code_values(x[u], 1, pv);
      const float2 c = code_values(x[u], 2, pv), d = code_values(x[u], 3, pv);
      o[u] = make_uint4(finite2(a.x, b.x, T{}), finite2(c.x, d.x, T{}), finite2(a.y, b.y, T{}), finite2(c.y, d.y, T{}));
    }
    for (int j = 0; j < cs.n; ++j) {
      uint4* dst = reinterpret_cast<uint4*>((kv ? p.dst.v : p.dst.k) + target_row(j) * D);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (tid + u * kCopyThreads < n * R::W) __stcs(dst + tid + u * kCopyThreads, o[u]);
    }
  }
  if (sidx == 0) {
    const int64_t from = p.src.st.off[cs.s] + r0;
    for (int i = tid; i < n; i += kCopyThreads) {
      const int32_t a = p.src.pos[from + i], b = p.src.orig[from + i];
      for (int j = 0; j < cs.n; ++j) {
        const int64_t to = p.dst.st.off[plan.targets[cs.first + j].s] + r0 + i;
        p.dst.pos[to] = a;
        p.dst.orig[to] = b;
      }
    }
  }
}

// The state that the next kernels read; a decode may do so as soon as this kernel's blocks have ended.
__device__ __forceinline__ void store_upload(const AppendImage& img, int bytes, uint4* dyn) {
  for (int i = threadIdx.x; i < bytes / 16; i += kCopyThreads) dyn[i] = img.v[i];
  __threadfence();
}

template <typename T, int D, int SB, int DB>
__global__ void __launch_bounds__(kCopyThreads) copy_kernel(CopyDev p, CopyPlan plan) {
  copy_block<T, D, SB, DB>(p, plan);
}

// The upload as a kernel parameter, which the first block stores in the workspace of the targets' cache.
template <typename T, int D, int SB, int DB>
__global__ void __launch_bounds__(kCopyThreads)
    copy_image_kernel(CopyDev p, const __grid_constant__ AppendImage img, int img_bytes, int sources, int targets, uint4* dyn) {
  if (blockIdx.x == 0) store_upload(img, img_bytes, dyn);
  const char* at = reinterpret_cast<const char*>(&img);
  const CopyPlan plan{reinterpret_cast<const CopySource*>(at + sources), reinterpret_cast<const CopyTarget*>(at + targets)};
  copy_block<T, D, SB, DB>(p, plan);
}

// Scores of the targets' streams, a block each: the source's or zero for rows [0, len) of a copy, zero for the slots up to
// len_old that no longer hold a row.
__device__ __forceinline__ void score_block(const CopyDev& p, const CopyTarget& t, bool copies) {
  const int sidx = blockIdx.x % (p.g.M * p.g.H), h = sidx % p.g.H, m = sidx / p.g.H;
  float* to = p.dst.scores + stream_row0(p.g, p.dst, m, h, t.s);
  if (copies) {
    const float* from = p.src.scores ? p.src.scores + stream_row0(p.g, p.src, m, h, t.src) : nullptr;
    for (int i = threadIdx.x; i < t.len; i += kCopyThreads) to[i] = from ? from[i] : 0.f;
  }
  for (int i = t.len + threadIdx.x; i < t.len_old; i += kCopyThreads) to[i] = 0.f;
}

__global__ void __launch_bounds__(kCopyThreads) copy_scores_kernel(CopyDev p, const CopyTarget* targets, int copies) {
  score_block(p, targets[blockIdx.x / (p.g.M * p.g.H)], copies != 0);
}

__global__ void __launch_bounds__(kCopyThreads)
    drop_image_kernel(CopyDev p, const __grid_constant__ AppendImage img, int img_bytes, int targets, uint4* dyn) {
  pdl_wait();  // a decode before it lets it start and still reads the state
  if (blockIdx.x == 0) store_upload(img, img_bytes, dyn);
  if (p.dst.scores == nullptr) return;
  const CopyTarget* t = reinterpret_cast<const CopyTarget*>(reinterpret_cast<const char*>(&img) + targets);
  score_block(p, t[blockIdx.x / (p.g.M * p.g.H)], false);
}

template <typename T, int D, int SB, int DB>
cudaError_t launch_t(const CopyDev& p, const CopyArgs& a, cudaStream_t stream) {
  const int64_t blocks = a.n_chunks * p.g.M * 2 * p.g.H;
  const char* dyn = static_cast<const char*>(a.dyn);
  if (a.img)
    copy_image_kernel<T, D, SB, DB><<<(unsigned)blocks, kCopyThreads, 0, stream>>>(
        p, *a.img, (int)a.img_bytes, (int)a.sources, (int)a.targets, static_cast<uint4*>(a.dyn));
  else
    copy_kernel<T, D, SB, DB><<<(unsigned)blocks, kCopyThreads, 0, stream>>>(
        p, {reinterpret_cast<const CopySource*>(dyn + a.sources), reinterpret_cast<const CopyTarget*>(dyn + a.targets)});
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_bits(const CopyDev& p, const CopyArgs& a, cudaStream_t stream) {
  const bool bf16 = p.g.dtype == 1;  // between equal bits the type does not matter
  if (a.src.bits == 16 && a.dst.bits == 16) return launch_t<F16T, D, 16, 16>(p, a, stream);
  if (a.src.bits == 4 && a.dst.bits == 4) return launch_t<F16T, D, 4, 4>(p, a, stream);
  if (a.src.bits == 16) return bf16 ? launch_t<BF16T, D, 16, 4>(p, a, stream) : launch_t<F16T, D, 16, 4>(p, a, stream);
  return bf16 ? launch_t<BF16T, D, 4, 16>(p, a, stream) : launch_t<F16T, D, 4, 16>(p, a, stream);
}

}  // namespace

cudaError_t launch_copy(const Geometry& g, const CopyArgs& a, cudaStream_t stream, int* launched) {
  *launched = 0;
  if (a.n_chunks <= 0) return launch_drop(g, a, stream, launched);
  const CopyDev p{g, a.src, a.dst, (int)a.n_chunks, a.n_sources};
  cudaError_t e = cudaErrorInvalidValue;
  switch (g.D) {
    case 64:
      e = launch_bits<64>(p, a, stream);
      break;
    case 80:
      e = launch_bits<80>(p, a, stream);
      break;
    case 96:
      e = launch_bits<96>(p, a, stream);
      break;
    case 128:
      e = launch_bits<128>(p, a, stream);
      break;
  }
  if (e != cudaSuccess) return e;
  *launched = 1;
  if (!a.dst.scores) return cudaSuccess;
  copy_scores_kernel<<<(unsigned)((int64_t)a.n_targets * g.M * g.H), kCopyThreads, 0, stream>>>(
      p, reinterpret_cast<const CopyTarget*>(static_cast<const char*>(a.dyn) + a.targets), 1);
  e = cudaGetLastError();
  if (e == cudaSuccess) *launched = 2;
  return e;
}

cudaError_t launch_drop(const Geometry& g, const CopyArgs& a, cudaStream_t stream, int* launched) {
  *launched = 0;
  const CopyDev p{g, a.src, a.dst, 0, 0};
  const unsigned blocks = a.dst.scores ? (unsigned)((int64_t)a.n_targets * g.M * g.H) : 1;
  if (a.img) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(kCopyThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, drop_image_kernel, p, *a.img, (int)a.img_bytes, (int)a.targets,
                                             static_cast<uint4*>(a.dyn));
    if (e != cudaSuccess) return e;
  } else if (a.dst.scores) {
    copy_scores_kernel<<<blocks, kCopyThreads, 0, stream>>>(
        p, reinterpret_cast<const CopyTarget*>(static_cast<const char*>(a.dyn) + a.targets), 0);
  } else {
    return cudaSuccess;
  }
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) *launched = 1;
  return e;
}

}  // namespace kvc
