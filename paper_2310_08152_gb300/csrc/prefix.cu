// Decode of sequences that share a prefix: a kernel for the rows that they share, and one for each sequence's own rows,
// which joins the two.
//
// prefix_kernel.  The samples of one prompt have the prompt's rows in common.  A decode of each on its own reads those rows once per
// sample; here one CTA takes the queries of up to 32 samples of a (layer, head) against a run of the prefix's rows, so
// that the rows are read once for all of them, and leaves for each sample the part's maximum, sum and unscaled output
//   m = max z_i,  l = sum 2^(z_i - m),  O = sum 2^(z_i - m) v_i,   z_i = scale log2(e) <q, k_i>,
// which own_kernel joins with the sample's own rows.
//
// The queries are the M rows of 16 x 8 x 16 matrix instructions: with the paper's 8 samples of a prompt the work is that
// of one 16-row tile, an eighth of the smallest tile of the tcgen05 instructions, and P stays in registers between the
// two products.  The warps share a CTA's keys; each keeps its own online softmax and
// the results are merged in shared memory at the end.  (More than 32 samples: prefix_tc.cu.)  Tiles of 64 rows come through a ring of two or three stages with 16-byte
// asynchronous copies into rows padded by 16 bytes, which keeps the matrix loads free of bank conflicts at every d_head.
//
// Precision.  q.k is exact in its products and summed in 32 bits; a rotated query, and P, go as two 16-bit parts in f16 (22
// bits) and three in bf16 (24), for the output is in 32 bits.  (With two of bf16 its error was 2.3e-6 where 32-bit
// arithmetic leaves 4e-7.)  P's reference is 2^6 to 2^14 below the running maximum, which keeps f16's low part out of its
// subnormal range and makes rescaling rare.  The tensor cores cut what they add rather than round it, which over thousands
// of rows adds up (29,706 rows, 2,048 into a sum: 5.5e-6): here they sum 16 rows at a time, and the sums are added outside;
// and a logit's small parts come before its large one (after it: 2.1e-6 at d_head 128 in bf16, 7e-7 so).
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <type_traits>

#include "device_common.cuh"
#include "kernels.hpp"
#include "tensor_core.cuh"

namespace kvc {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kThreads = 128;
constexpr int kKeys = 64;  // rows per tile

// R = 16 MT queries per CTA: MT 16-row tiles in each of four warps, which share the keys.
// NQ 16-bit parts of a query.
template <int D, int MT, int NQ>
struct PxCfg {
  static constexpr int R = 16 * MT;
  static constexpr int KW = kThreads / 32;
  static constexpr int KG = kKeys / KW / 16;  // 16-key groups per warp and tile
  static constexpr int RS = D * 2 + 16;       // bytes of a row in shared memory
  static constexpr int TILE = kKeys * RS;
  static constexpr int S = MT == 1 ? 2 : 3;   // stages: two leave room for a fourth CTA per SM
  static constexpr int OFF_Q = 2 * S * TILE;
  static constexpr int SMEM = OFF_Q + NQ * R * RS;
  static constexpr int PO = D + 4;
  static_assert(KW * R * PO * 4 <= OFF_Q, "the warps' results fit in the stages");
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}

template <typename T>
struct Mma;
template <>
struct Mma<F16T> {
  static __device__ __forceinline__ void go(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Mma<BF16T> {
  static __device__ __forceinline__ void go(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

template <typename T, int D, int MT, int NQ>
__global__ void __launch_bounds__(kThreads, D > 96 && MT > 1 ? 2 : MT == 1 && D < 96 ? 4 : 3) prefix_kernel(PrefixArgs p) {
  using C = PxCfg<D, MT, NQ>;
  constexpr int WM = MT, KG = C::KG, CH = D / 8, NP = kFullParts<T>;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kw = warp;
  const uint32_t s0 = smem_addr(smem);
  pdl_wait();               // q and the prefix's rows come from earlier kernels
  pdl_launch_dependents();  // the own rows' decode may start: what it reads before its wait is complete by now
  const int lh = (int)(blockIdx.x / (unsigned)p.n_units);
  const PrefixUnit un = p.units[blockIdx.x - lh * p.n_units];
  const int layer = lh / p.H, h = lh - layer * p.H;
  const int64_t row0 = (int64_t)(p.layer + layer) * p.H * p.C + p.st.seq_row0[un.s] + (int64_t)h * p.st.cap[un.s] + un.key0;
  const int n_keys = un.key1 - un.key0, n_tiles = (n_keys + kKeys - 1) / kKeys;
  const uint16_t* gk = p.k + row0 * D;
  const uint16_t* gv = p.v + row0 * D;
  auto load = [&](int t) {  // tile t into its stage; rows past the last one as zeros
    if (t < n_tiles) {
      const uint32_t dst = s0 + (t % C::S) * 2 * C::TILE;
#pragma unroll
      for (int x = tid; x < kKeys * CH; x += kThreads) {
        const int r = x / CH, c = x % CH;
        const int key = t * kKeys + r;
        const bool in = key < n_keys;
        const int64_t e = in ? (int64_t)key * D + c * 8 : 0;
        cp16(dst + r * C::RS + c * 16, gk + e, in ? 16u : 0u);
        cp16(dst + C::TILE + r * C::RS + c * 16, gv + e, in ? 16u : 0u);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int t = 0; t < C::S - 1; ++t) load(t);

  // the queries, rotated where the cache's keys are
  for (int x = tid; x < C::R * CH; x += kThreads) {
    const int r = x / CH, c = x % CH;
    uint32_t part[NQ][4];
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) part[i][e] = 0;
    if (r < un.n_mem) {
      const int s = p.members[un.mem0 + r];
      const uint16_t* q = p.q + (int64_t)layer * p.q_stride + ((int64_t)s * p.H + h) * D;
      query_chunk<T, NQ>(q, c, p.rot, NQ > 1 ? p.ds[s].qpos : 0, p.st.rope_g, part);
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i)
      *reinterpret_cast<uint4*>(smem + C::OFF_Q + (i * C::R + r) * C::RS + c * 16) =
          make_uint4(part[i][0], part[i][1], part[i][2], part[i][3]);
  }

  // matrix addresses of this lane: A and V^T tiles take rows lane % 16 and the column half lane / 16; K tiles the keys
  // lane % 8 + 8 (lane / 16) and the column half lane / 8 % 2
  const uint32_t a_off = (lane & 15) * C::RS + (lane >> 4) * 16;
  const uint32_t k_off = ((lane & 7) + (lane >> 4) * 8) * C::RS + (lane >> 3 & 1) * 16;
  const uint32_t q_addr = s0 + C::OFF_Q + a_off;
  float o[WM][D / 8][4];
  float m[WM][2], l[WM][2];
#pragma unroll
  for (int i = 0; i < WM; ++i) {
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
    m[i][0] = m[i][1] = -INFINITY;
    l[i][0] = l[i][1] = 0.f;
  }
  for (int t = 0; t < n_tiles; ++t) {
    asm volatile("cp.async.wait_group %0;" ::"n"(C::S - 2) : "memory");
    __syncthreads();  // tile t is here for every warp, and tile t - 1 is read
    load(t + C::S - 1);
    const uint32_t kt = s0 + (t % C::S) * 2 * C::TILE + kw * KG * 16 * C::RS, vt = kt + C::TILE;
    float z[WM][KG * 2][4];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int n = 0; n < KG * 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[i][n][e] = 0.f;
    // z += the product of parts [x0, x1); the small ones first, which the tensor cores would cut at the whole sum's last bit
    auto add_parts = [&](auto x0c, auto x1c) {
      constexpr int X0 = decltype(x0c)::value, NX = decltype(x1c)::value - X0;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t a[NX][WM][4];
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
          for (int i = 0; i < WM; ++i) ldsm4(a[x][i], q_addr + ((X0 + x) * C::R + i * 16) * C::RS + kk * 32);
#pragma unroll
        for (int g = 0; g < KG; ++g) {
          uint32_t b[4];
          ldsm4(b, kt + g * 16 * C::RS + k_off + kk * 32);
#pragma unroll
          for (int x = NX - 1; x >= 0; --x)
#pragma unroll
            for (int i = 0; i < WM; ++i) {
              Mma<T>::go(z[i][2 * g], a[x][i], b[0], b[1]);
              Mma<T>::go(z[i][2 * g + 1], a[x][i], b[2], b[3]);
            }
        }
      }
    };
    if constexpr (NQ > 1) add_parts(std::integral_constant<int, 1>{}, std::integral_constant<int, NQ>{});
    add_parts(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
    const int left = n_keys - t * kKeys - kw * KG * 16;  // the warp's keys of this tile that exist
    const bool ragged = left < KG * 16;
    bool moved = false;
    float scale_o[WM][2];
#pragma unroll
    for (int i = 0; i < WM; ++i) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        float mx = -INFINITY;
#pragma unroll
        for (int n = 0; n < KG * 2; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = z[i][n][2 * hh + e] * p.c2;
            if (ragged && n * 8 + (lane & 3) * 2 + e >= left) x = -INFINITY;
            z[i][n][2 * hh + e] = x;
            mx = fmaxf(mx, x);
          }
        mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, 2));
        scale_o[i][hh] = 1.f;
        if (mx > m[i][hh] + 14.f) {
          const float to = mx - 6.f;
          scale_o[i][hh] = m[i][hh] == -INFINITY ? 0.f : ex2(m[i][hh] - to);
          m[i][hh] = to;
          moved = true;
        }
      }
    }
    if (__any_sync(kFull, moved)) {
#pragma unroll
      for (int i = 0; i < WM; ++i) {
        l[i][0] *= scale_o[i][0];
        l[i][1] *= scale_o[i][1];
#pragma unroll
        for (int n = 0; n < D / 8; ++n) {
          o[i][n][0] *= scale_o[i][0];
          o[i][n][1] *= scale_o[i][0];
          o[i][n][2] *= scale_o[i][1];
          o[i][n][3] *= scale_o[i][1];
        }
      }
    }
#pragma unroll
    for (int g = 0; g < KG; ++g) {
      uint32_t pp[NP][WM][4];
#pragma unroll
      for (int i = 0; i < WM; ++i) {
#pragma unroll
        for (int f = 0; f < 4; ++f) {  // the A tile: rows 0, 8, 0, 8 of keys 0, 0, 8, 8
          const int n = 2 * g + (f >> 1), hh = f & 1;
          const float mu = m[i][hh] == -INFINITY ? 0.f : m[i][hh];
          const float p0 = ex2(z[i][n][2 * hh] - mu), p1 = ex2(z[i][n][2 * hh + 1] - mu);
          l[i][hh] += p0 + p1;
          uint32_t part[NP];
          split_parts<T, NP>(p0, p1, part);
#pragma unroll
          for (int x = 0; x < NP; ++x) pp[x][i][f] = part[x];
        }
      }
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t b[4];
        ldsm4t(b, vt + g * 16 * C::RS + a_off + n * 32);
#pragma unroll
        for (int i = 0; i < WM; ++i) {
          float sum[2][4] = {};
#pragma unroll
          for (int x = NP - 1; x >= 0; --x) {
            Mma<T>::go(sum[0], pp[x][i], b[0], b[1]);
            Mma<T>::go(sum[1], pp[x][i], b[2], b[3]);
          }
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              float* at = &o[i][2 * n + y][e];
              const float2 v = __fadd2_rn(make_float2(at[0], at[1]), make_float2(sum[y][e], sum[y][e + 1]));
              at[0] = v.x;
              at[1] = v.y;
            }
        }
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();  // every tile is read: the stages take the warps' results
  float* res = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      float s = l[i][hh];
      s += __shfl_xor_sync(kFull, s, 1);
      s += __shfl_xor_sync(kFull, s, 2);
      float* to = res + ((int64_t)kw * C::R + i * 16 + hh * 8 + (lane >> 2)) * C::PO;
      if ((lane & 3) == 0) {
        to[0] = m[i][hh];
        to[1] = s;
      }
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
        *reinterpret_cast<float2*>(to + 4 + n * 8 + (lane & 3) * 2) = make_float2(o[i][n][2 * hh], o[i][n][2 * hh + 1]);
    }
  __syncthreads();
  // the warps of one query joined, a float4 of its part per thread
  for (int x = tid; x < un.n_mem * (C::PO / 4); x += kThreads) {
    const int r = x / (C::PO / 4), c = x % (C::PO / 4);
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < C::KW; ++w) M = fmaxf(M, res[(w * C::R + r) * C::PO]);
    const float Mu = M == -INFINITY ? 0.f : M;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < C::KW; ++w) {
      const float* from = res + (w * C::R + r) * C::PO;
      const float e = ex2(from[0] - Mu);
      if (c == 0) {
        sum.y += from[1] * e;
      } else {
        const float4 v = *reinterpret_cast<const float4*>(from + 4 * c);
        sum.x += v.x * e;
        sum.y += v.y * e;
        sum.z += v.z * e;
        sum.w += v.w * e;
      }
    }
    if (c == 0) sum.x = M;
    const int s = p.members[un.mem0 + r];
    float* to = p.parts + (((int64_t)layer * p.n_parts + p.split0[s] + un.split) * p.H + h) * C::PO;
    *reinterpret_cast<float4*>(to + 4 * c) = sum;
  }
}

template <typename T, int D, int MT, int NQ>
cudaError_t prefix_occ(int dev, int* occ) {
  using C = PxCfg<D, MT, NQ>;
  static std::atomic<int> found[64];
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  int o = found[dev].load(std::memory_order_acquire);
  if (o == 0) {
    cudaError_t e = cudaFuncSetAttribute(prefix_kernel<T, D, MT, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&o, prefix_kernel<T, D, MT, NQ>, kThreads, C::SMEM);
    if (e != cudaSuccess) return e;
    if (o < 1) o = 1;
    found[dev].store(o, std::memory_order_release);
  }
  *occ = o;
  return cudaSuccess;
}

// ---------------------------------------------------------------------------------------------
// The own rows, and the join
// ---------------------------------------------------------------------------------------------
// A sample has a few own rows, at first one, and there are as many segments as samples, heads and layers: a warp takes a
// whole segment (WPS = 1), or four warps share one where the segments are few or long (WPS = 4).  LPR lanes share a row,
// so that a load instruction takes whole sectors of RPI rows, straight into registers; U steps of K and V rows are under
// way at a time.  The row groups' results meet in shared memory, then the warps', then the prefix's parts.
template <int D>
struct OwnLanes {
  static constexpr int CH = D / 8;
  static constexpr int LPR = D == 80 ? 2 : D == 96 ? 4 : 8;
  static constexpr int NV = CH / LPR;
  static constexpr int RPI = 32 / LPR;
  static constexpr int U = D == 64 ? 4 : D == 80 ? 1 : 2;
  static constexpr int ROWS = U * RPI;
};
constexpr int kOwnWarps = 4;
// SCORED: the decode of many short segments that adds each row's weight to its score, no prefix.  The logits (of up to
// kOwnHeld rows) stay in shared memory until the segment's maximum and sum are known, so K and V are read once; each score
// takes one addition of this call.  Bound by the bytes of K, V and the scores.
constexpr int kOwnHeld = 1024;

template <typename T, int D, int WPS, bool SCORED>
__global__ void __launch_bounds__(kOwnWarps * 32, 4) own_kernel(OwnArgs a) {
  using L = OwnLanes<D>;
  constexpr int NV = L::NV, U = L::U, QPL = (D + 31) / 32, PO = D + 4;
  __shared__ __align__(16) float s_q[kOwnWarps][D];
  __shared__ __align__(16) float s_o[kOwnWarps][L::RPI][D];  // the row groups' columns; the first row of a warp's: its result
  __shared__ float s_ml[kOwnWarps][2];
  __shared__ float s_z[SCORED ? kOwnWarps : 1][SCORED ? kOwnHeld : 1];
  static_assert(!SCORED || WPS == 1, "a warp has its segment's logits");
  const PrefixArgs& p = a.px;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (!a.early) pdl_wait();  // else whatever the prefix kernel waited for is complete, and it writes only the parts
  pdl_launch_dependents();
  const int H = p.H;
  const int64_t seg = ((int64_t)blockIdx.x * kOwnWarps + warp) / WPS, per_layer = (int64_t)a.b * H;
  const int sub = warp % WPS;
  const bool live = seg < per_layer * p.n_layers;
  const int layer = live ? (int)(seg / per_layer) : 0;
  const int w = live ? (int)(seg - layer * per_layer) : 0, s = w / H, h = w - s * H;
  const DState d = p.ds[s];
  const int len = live ? d.len : 0;  // 0: the sequence has no token
  const int n_split = SCORED || d.is_cl ? 0 : p.n_split[s];
  const int64_t row0 = (int64_t)(p.layer + layer) * H * p.C + p.st.seq_row0[s] + (int64_t)h * p.st.cap[s];
  float* qs = s_q[warp];
  const float* part = SCORED ? nullptr : p.parts + (((int64_t)layer * p.n_parts + p.split0[s]) * H + h) * PO;
  // the first part is there already where this kernel did not start early: its loads are under way with the rows'
  float M0 = -INFINITY, L0 = 0.f, O0[QPL];
  auto load_part = [&]() {
    M0 = __ldcg(part);
    L0 = __ldcg(part + 1);
#pragma unroll
    for (int k = 0; k < QPL; ++k) O0[k] = lane + 32 * k < D ? __ldcg(part + 4 + lane + 32 * k) : 0.f;
  };
  if (!a.early && n_split > 0 && sub == 0) load_part();
  if (len > 0) {
    const uint16_t* q = p.q + (int64_t)layer * p.q_stride + (int64_t)w * D;
    const int half = p.rot / 2;
#pragma unroll
    for (int j = 0; j < QPL; ++j) {
      const int c = lane + 32 * j;
      if (c < D) {
        if (c >= p.rot) {
          qs[c] = T::f1(q[c]) * p.c2;
        } else if (c < half) {
          float sn, cs;
          rope_sincos_full(d.qpos, p.st.rope_g[c], &sn, &cs);
          const float x = T::f1(q[c]), y = T::f1(q[c + half]);
          qs[c] = (x * cs - y * sn) * p.c2;
          qs[c + half] = (y * cs + x * sn) * p.c2;
        }
      }
    }
  }
  __syncwarp();
  const int grp = lane / L::LPR, tl = lane % L::LPR;
  float2 o[NV * 4];
#pragma unroll
  for (int e = 0; e < NV * 4; ++e) o[e] = make_float2(0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  for (int r0 = d.begin + sub * L::ROWS; r0 < len; r0 += WPS * L::ROWS) {
    uint4 k[U][NV], v[U][NV];
    bool ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * L::RPI + grp;
      ok[u] = r < len && (r < d.mask_lo || r >= d.mask_hi);
      const uint4* kr = reinterpret_cast<const uint4*>(p.k + (row0 + r) * D) + tl;
      const uint4* vr = reinterpret_cast<const uint4*>(p.v + (row0 + r) * D) + tl;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        k[u][i] = v[u][i] = make_uint4(0, 0, 0, 0);
        if (ok[u]) k[u][i] = __ldcs(kr + i * L::LPR);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (ok[u]) v[u][i] = __ldcs(vr + i * L::LPR);
    }
    float z[U], mn = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float2 acc0 = make_float2(0.f, 0.f), acc1 = acc0;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float4 qa = *reinterpret_cast<const float4*>(qs + (i * L::LPR + tl) * 8);
        const float4 qb = *reinterpret_cast<const float4*>(qs + (i * L::LPR + tl) * 8 + 4);
        acc0 = __ffma2_rn(make_float2(qa.x, qa.y), T::f2(k[u][i].x), acc0);
        acc1 = __ffma2_rn(make_float2(qa.z, qa.w), T::f2(k[u][i].y), acc1);
        acc0 = __ffma2_rn(make_float2(qb.x, qb.y), T::f2(k[u][i].z), acc0);
        acc1 = __ffma2_rn(make_float2(qb.z, qb.w), T::f2(k[u][i].w), acc1);
      }
      z[u] = (acc0.x + acc1.x) + (acc0.y + acc1.y);
#pragma unroll
      for (int off = L::LPR / 2; off >= 1; off >>= 1) z[u] += __shfl_xor_sync(kFull, z[u], off);
      if (!ok[u]) z[u] = -INFINITY;
      if constexpr (SCORED) {
        const int x = r0 + u * L::RPI + grp - d.begin;
        if (tl == 0 && x < kOwnHeld) s_z[warp][x] = z[u];
      }
      mn = fmaxf(mn, z[u]);
    }
    const float mu = mn == -INFINITY ? 0.f : mn;
    const float alpha = exp2f(m - mu);
    l *= alpha;
#pragma unroll
    for (int e = 0; e < NV * 4; ++e) o[e] = __fmul2_rn(o[e], make_float2(alpha, alpha));
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float pk = exp2f(z[u] - mu);
      const float2 p2 = make_float2(pk, pk);
      l += pk;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        o[i * 4 + 0] = __ffma2_rn(p2, T::f2(v[u][i].x), o[i * 4 + 0]);
        o[i * 4 + 1] = __ffma2_rn(p2, T::f2(v[u][i].y), o[i * 4 + 1]);
        o[i * 4 + 2] = __ffma2_rn(p2, T::f2(v[u][i].z), o[i * 4 + 2]);
        o[i * 4 + 3] = __ffma2_rn(p2, T::f2(v[u][i].w), o[i * 4 + 3]);
      }
    }
    m = mn;
  }
  // the row groups joined
  float M = m;
#pragma unroll
  for (int off = 16; off >= L::LPR; off >>= 1) M = fmaxf(M, __shfl_xor_sync(kFull, M, off));
  const float e = exp2f(m - (M == -INFINITY ? 0.f : M));
  float Ls = l * e;
#pragma unroll
  for (int off = 16; off >= L::LPR; off >>= 1) Ls += __shfl_xor_sync(kFull, Ls, off);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float4* dst = reinterpret_cast<float4*>(&s_o[warp][grp][(i * L::LPR + tl) * 8]);
    dst[0] = make_float4(o[i * 4].x * e, o[i * 4].y * e, o[i * 4 + 1].x * e, o[i * 4 + 1].y * e);
    dst[1] = make_float4(o[i * 4 + 2].x * e, o[i * 4 + 2].y * e, o[i * 4 + 3].x * e, o[i * 4 + 3].y * e);
  }
  __syncwarp();
  float O[QPL];
#pragma unroll
  for (int j = 0; j < QPL; ++j) {
    O[j] = 0.f;
    const int c = lane + 32 * j;
    if (c < D)
#pragma unroll
      for (int g = 0; g < L::RPI; ++g) O[j] += s_o[warp][g][c];
  }
  if constexpr (WPS > 1) {  // the warps of a segment
    __syncwarp();
    if (lane == 0) {
      s_ml[warp][0] = M;
      s_ml[warp][1] = Ls;
    }
#pragma unroll
    for (int j = 0; j < QPL; ++j)
      if (lane + 32 * j < D) s_o[warp][0][lane + 32 * j] = O[j];
    __syncthreads();
    if (sub == 0) {
      float Mx = M;
#pragma unroll
      for (int x = 1; x < WPS; ++x) Mx = fmaxf(Mx, s_ml[warp + x][0]);
      const float Mu = Mx == -INFINITY ? 0.f : Mx;
      const float e0 = exp2f(M - Mu);
      Ls *= e0;
#pragma unroll
      for (int j = 0; j < QPL; ++j) O[j] *= e0;
#pragma unroll
      for (int x = 1; x < WPS; ++x) {
        const float ex = exp2f(s_ml[warp + x][0] - Mu);
        Ls += s_ml[warp + x][1] * ex;
#pragma unroll
        for (int j = 0; j < QPL; ++j)
          if (lane + 32 * j < D) O[j] += s_o[warp + x][0][lane + 32 * j] * ex;
      }
      M = Mx;
    }
  }
  if constexpr (SCORED) {
    if (len > 0) {
      const float Mu = M == -INFINITY ? 0.f : M, inv = 1.f / Ls;
      float* sc = a.scores + (int64_t)(p.layer + layer) * H * p.C + p.st.seq_row0[s] + (int64_t)h * p.st.cap[s] + d.begin;
      for (int x = lane; x < len - d.begin; x += 32) {  // written by this warp, before the barriers above
        const int row = d.begin + x;
        if (row >= d.mask_lo && row < d.mask_hi) continue;  // a hidden row gets nothing, not even a NaN
        const float w = exp2f(s_z[warp][x] - Mu) * inv;
        if (w != 0.f) atomicAdd(sc + x, w);
      }
    }
  }
  if (a.early) pdl_wait();  // the parts; every thread of the grid waits, so that it never ends before the prefix's
  if (len == 0 || sub != 0) return;
  if (a.early && n_split > 0) load_part();
  const int64_t step = (int64_t)H * PO;
  for (int j = 0; j < n_split; ++j) {
    if (j > 0) {
      part += step;
      load_part();
    }
    const float Mn = fmaxf(M, M0), Mu = Mn == -INFINITY ? 0.f : Mn;
    const float eo = exp2f(M - Mu), ej = exp2f(M0 - Mu);
    Ls = Ls * eo + L0 * ej;
#pragma unroll
    for (int k = 0; k < QPL; ++k) O[k] = O[k] * eo + O0[k] * ej;
    M = Mn;
  }
  const float inv = 1.f / Ls;
  float* out = a.out + (int64_t)layer * a.out_stride + (int64_t)w * D;
#pragma unroll
  for (int k = 0; k < QPL; ++k)
    if (lane + 32 * k < D) out[lane + 32 * k] = O[k] * inv;
}

template <typename T, int D, int WPS, bool SCORED>
cudaError_t launch_own_t(const OwnArgs& a, int64_t segs, cudaStream_t stream, DecodePlan* plan) {
  *plan = {2, (int)(segs * WPS), OwnLanes<D>::ROWS, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((segs * WPS + kOwnWarps - 1) / kOwnWarps));
  cfg.blockDim = dim3(kOwnWarps * 32);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SCORED || a.early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, own_kernel<T, D, WPS, SCORED>, a);
}

template <typename F>
cudaError_t by_shape(const Geometry& g, int rows, F&& f) {
  auto mt = [&](auto tc, auto dc, auto rc) {
    if (rows <= 16) return f(tc, dc, std::integral_constant<int, 1>{}, rc);
    return f(tc, dc, std::integral_constant<int, 2>{}, rc);
  };
  auto rot = [&](auto tc, auto dc) { return g.rot > 0 ? mt(tc, dc, std::true_type{}) : mt(tc, dc, std::false_type{}); };
  auto dt = [&](auto dc) { return g.dtype == 1 ? rot(BF16T{}, dc) : rot(F16T{}, dc); };
  switch (g.D) {
    case 64:
      return dt(std::integral_constant<int, 64>{});
    case 80:
      return dt(std::integral_constant<int, 80>{});
    case 96:
      return dt(std::integral_constant<int, 96>{});
    case 128:
      return dt(std::integral_constant<int, 128>{});
    default:
      return cudaErrorInvalidValue;
  }
}

}  // namespace

int prefix_rows(int group) { return group <= 16 ? 16 : group <= 32 ? 32 : kPrefixTcRows; }

cudaError_t prefix_ctas_per_sm(const Geometry& g, int device, int rows, int* occ) {
  if (rows == kPrefixTcRows) {
    *occ = 1;
    return cudaSuccess;
  }
  return by_shape(g, rows, [&](auto t, auto d, auto m, auto r) {
    using T = decltype(t);
    return prefix_occ<T, decltype(d)::value, decltype(m)::value, (decltype(r)::value ? kFullParts<T> : 1)>(device, occ);
  });
}

cudaError_t launch_prefix(const Geometry& g, const PrefixArgs& a, int device, int rows, cudaStream_t stream) {
  if (a.n_units <= 0) return cudaSuccess;
  return by_shape(g, rows, [&](auto t, auto d, auto m, auto r) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value, MT = decltype(m)::value;
    constexpr int NQ = decltype(r)::value ? kFullParts<T> : 1;
    int occ = 0;
    const cudaError_t e = prefix_occ<T, D, MT, NQ>(device, &occ);  // sets the kernel's shared memory
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((int64_t)a.n_units * g.H * a.n_layers));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = PxCfg<D, MT, NQ>::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, prefix_kernel<T, D, MT, NQ>, a);
  });
}

cudaError_t launch_own(const Geometry& g, const OwnArgs& a, int64_t max_segment, int num_sms, cudaStream_t stream,
                       DecodePlan* plan) {
  const int64_t segs = (int64_t)a.px.n_layers * a.b * g.H;
  const bool share = segs <= 16 * (int64_t)num_sms || max_segment > 1024;
  return by_shape(g, 16, [&](auto t, auto d, auto, auto) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return share ? launch_own_t<T, D, 4, false>(a, segs, stream, plan) : launch_own_t<T, D, 1, false>(a, segs, stream, plan);
  });
}

// A warp for each segment where there are many short ones, else the CTAs of the scored decode.  us with CTAs -> with warps,
// f16, d_head 64: 12,288 segments of 95 rows 80 -> 51 (what they read and write would take 45.5), of 200 rows 129 -> 100,
// of 400 rows 224 -> 187, of 700 rows 335 -> 326, of 1,024 rows 463 -> 485; d_head 128, bf16: of 120 rows 139 -> 127,
// 6,144 of 700 rows 318 -> 343.  Fewer segments leave warps without work: 1,280 of 300 rows 20.6 -> 21.2 (d_head 128: 35.4
// -> 44.3), 512 of 100 rows 4.7 -> 6.9.
bool own_scored_takes(int64_t n_segments, int64_t rows, int64_t max_segment, int num_sms) {
  return max_segment <= kOwnHeld && rows <= 400 * n_segments && n_segments >= 16 * (int64_t)num_sms;
}

cudaError_t launch_own_scored(const Geometry& g, const OwnArgs& a, cudaStream_t stream, DecodePlan* plan) {
  return by_shape(g, 16, [&](auto t, auto d, auto, auto) {
    return launch_own_t<decltype(t), decltype(d)::value, 1, true>(a, (int64_t)a.px.n_layers * a.b * g.H, stream, plan);
  });
}

}  // namespace kvc
