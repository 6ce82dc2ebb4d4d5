// Kernels of a cache whose rows are held in 4 bits (packed.cuh has the format).
//
//   packed_append_kernel  new tokens' K/V rows, K rotated and rounded as the 16-bit append does it, into codes and pairs
//   packed_move_kernel    the row moves of a compaction
//   packed_decode_kernel  the decode over the codes
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernels.hpp"
#include "packed.cuh"

namespace kvc {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;

// ---------------------------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------------------------
// A block takes (layer, group of TG tokens) units; a lane takes eight columns of a row, the four lanes of a group of
// columns side by side.  The tokens of a unit come before the heads, so that a warp writes the rows of TG tokens, which are
// neighbours in a stream, together.
constexpr int kPackThreads = 256;
constexpr int kPackTokens = 4;

template <typename T, int D>
__device__ __forceinline__ void pack_units(const Geometry& g, const Static& st, const Buffers& buf, const PackedBuffers& pb,
                                           const TokPlan* plan, int64_t ntok, int64_t n_in, int m0, int n_layers, int tg,
                                           int write_meta, const uint16_t* __restrict__ k_in,
                                           const uint16_t* __restrict__ v_in) {
  using R = PackedRow<D>;
  __shared__ float2 rope_cs[kPackTokens][D / 2];  // (cos, sin) of the tokens' rotated pairs
  const int H = g.H, half = g.rot / 2;
  const int64_t groups = (ntok + tg - 1) / tg, n_units = groups * n_layers;
  const int n_items = 2 * H * tg * R::CP;
  for (int64_t u = blockIdx.x; u < n_units; u += gridDim.x) {
    const int l = (int)(u / groups);
    const int64_t t0 = (u - (int64_t)l * groups) * tg;
    const int nt = (int)min((int64_t)tg, ntok - t0);
    if (half > 0) {
      __syncthreads();  // the unit before is done with the table
      for (int i = threadIdx.x; i < nt * half; i += blockDim.x) {
        const int t = i / half, j = i - t * half;
        float sn, cs;
        rope_sincos(plan[t0 + t].pos, st.rope_g[j], &sn, &cs);
        rope_cs[t][j] = make_float2(cs, sn);
      }
      __syncthreads();
    }
    // a multiple of 32 for every warp: the lanes of a group reduce together
    for (int i = threadIdx.x; i < (n_items + 31) / 32 * 32; i += blockDim.x) {
      const int c = i % R::CP, j = i / R::CP, t = j % tg, hk = j / tg;
      const bool is_v = hk >= H;
      const int h = is_v ? hk - H : hk;
      const bool active = hk < 2 * H && t < nt && c < R::W;
      const TokPlan tp = plan[t0 + min(t, nt - 1)];
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (active) {
        const uint16_t* src = (is_v ? v_in : k_in) + (((int64_t)l * n_in + tp.in_tok) * H + h) * D;
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(src + 8 * c));
        const uint32_t av[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = T::f2(av[e]);
          x[2 * e] = f.x;
          x[2 * e + 1] = f.y;
        }
        if (!is_v && 8 * c < g.rot) {
          const bool first = 8 * c < half;
          const int p0 = first ? 8 * c : 8 * c - half;
          const uint4 b = __ldg(reinterpret_cast<const uint4*>(src + (first ? 8 * c + half : p0)));
          const uint32_t bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = T::f2(bv[e]);
            const float2 r0 = rope_cs[t][p0 + 2 * e], r1 = rope_cs[t][p0 + 2 * e + 1];
            const float y0 = first ? x[2 * e] * r0.x - f.x * r0.y : x[2 * e] * r0.x + f.x * r0.y;
            const float y1 = first ? x[2 * e + 1] * r1.x - f.y * r1.y : x[2 * e + 1] * r1.x + f.y * r1.y;
            x[2 * e] = T::f1(T::r(y0));
            x[2 * e + 1] = T::f1(T::r(y1));
          }
        }
      }
      uint32_t pair;
      const uint32_t word = pack8<T>(x, active, &pair);
      if (!active) continue;
      const int64_t row = (int64_t)(m0 + l) * H * g.C + st.seq_row0[tp.s] + (int64_t)h * st.cap[tp.s] + tp.row;
      reinterpret_cast<uint32_t*>(is_v ? pb.vc : pb.kc)[row * R::W + c] = word;
      if (c % 4 == 0) (is_v ? pb.vp : pb.kp)[row * R::G + c / 4] = pair;
    }
    if (write_meta && l == 0 && threadIdx.x < nt) {
      const TokPlan tp = plan[t0 + threadIdx.x];
      buf.pos[st.off[tp.s] + tp.row] = tp.pos;
      buf.orig[st.off[tp.s] + tp.row] = tp.orig;
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kPackThreads)
    packed_append_kernel(Geometry g, Static st, Buffers buf, PackedBuffers pb, const TokPlan* __restrict__ plan, int64_t ntok,
                         int64_t n_in, int m0, int n_layers, int tg, int write_meta, const uint16_t* __restrict__ k_in,
                         const uint16_t* __restrict__ v_in) {
  pack_units<T, D>(g, st, buf, pb, plan, ntok, n_in, m0, n_layers, tg, write_meta, k_in, v_in);
}

// The upload as a kernel parameter, as for the 16-bit append of a few tokens.
template <typename T, int D>
__global__ void __launch_bounds__(kPackThreads)
    packed_append_image_kernel(Geometry g, Static st, Buffers buf, PackedBuffers pb, const __grid_constant__ AppendImage img,
                               int img_bytes, int plan_off, uint4* dyn, int64_t ntok, int64_t n_in, int n_layers, int tg,
                               const uint16_t* __restrict__ k_in, const uint16_t* __restrict__ v_in) {
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < img_bytes / 16; i += blockDim.x) dyn[i] = img.v[i];
  pack_units<T, D>(g, st, buf, pb, reinterpret_cast<const TokPlan*>(reinterpret_cast<const char*>(&img) + plan_off), ntok,
                   n_in, 0, n_layers, tg, 1, k_in, v_in);
}

// ---------------------------------------------------------------------------------------------
// Row moves of a compaction: as the 16-bit rows', a block a (sequence, layer, K/V, head) stream that walks its destination
// rows upward, each chunk's loads ahead of its stores.  Codes go as 8-byte parts, pairs as words.
// ---------------------------------------------------------------------------------------------
constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 128;

template <int D>
__global__ void __launch_bounds__(kMoveThreads)
    packed_move_kernel(Geometry g, Static st, PackedBuffers pb, const AffSeq* __restrict__ aff, const int32_t* __restrict__ src_map) {
  using R = PackedRow<D>;
  constexpr int CPR = R::RB / 8;                             // parts of codes a row
  constexpr int UC = (kMoveRows * CPR + kMoveThreads - 1) / kMoveThreads;
  constexpr int UP = (kMoveRows * R::G + kMoveThreads - 1) / kMoveThreads;
  const int streams = g.M * 2 * g.H;
  const int sidx = blockIdx.x % streams;
  const int h = sidx % g.H, kv = (sidx / g.H) & 1, m = sidx / (2 * g.H);
  const AffSeq a = aff[blockIdx.x / streams];
  const int64_t row0 = (int64_t)m * g.H * g.C + st.seq_row0[a.s] + (int64_t)h * st.cap[a.s];
  uint2* codes = reinterpret_cast<uint2*>(kv ? pb.vc : pb.kc) + row0 * CPR;
  uint32_t* pairs = (kv ? pb.vp : pb.kp) + row0 * R::G;
  const int32_t* smap = src_map + st.off[a.s];
  struct Chunk {
    uint2 c[UC];
    uint32_t p[UP];
  };
  auto load = [&](int d0, Chunk& x) {
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const int i = threadIdx.x + u * kMoveThreads, r = i / CPR, row = d0 + r;
      if (r < kMoveRows && row < a.len_new) x.c[u] = codes[(int64_t)__ldg(smap + row) * CPR + i % CPR];
    }
#pragma unroll
    for (int u = 0; u < UP; ++u) {
      const int i = threadIdx.x + u * kMoveThreads, r = i / R::G, row = d0 + r;
      if (r < kMoveRows && row < a.len_new) x.p[u] = pairs[(int64_t)__ldg(smap + row) * R::G + i % R::G];
    }
  };
  Chunk now, next;
  int d0 = a.first_row;
  if (d0 >= a.len_new) return;
  load(d0, now);
  for (; d0 < a.len_new; d0 += kMoveRows) {
    if (d0 + kMoveRows < a.len_new) load(d0 + kMoveRows, next);
    __syncthreads();  // a kept row only moves down: the next chunk's sources lie above this chunk's destinations
#pragma unroll
    for (int u = 0; u < UC; ++u) {
      const int i = threadIdx.x + u * kMoveThreads, r = i / CPR, row = d0 + r;
      if (r < kMoveRows && row < a.len_new) codes[(int64_t)row * CPR + i % CPR] = now.c[u];
    }
#pragma unroll
    for (int u = 0; u < UP; ++u) {
      const int i = threadIdx.x + u * kMoveThreads, r = i / R::G, row = d0 + r;
      if (r < kMoveRows && row < a.len_new) pairs[(int64_t)row * R::G + i % R::G] = now.p[u];
    }
    now = next;
  }
}

// ---------------------------------------------------------------------------------------------
// Decode: out = sum_j softmax_j(scale <q, k_j>) v_j over the rows that the query sees, with k_j = lo + step c_j a group of
// columns:  <q, k_j> = sum over the groups of step <q, c_j> + lo sum(q).  A block a (layer, sequence, head); a row a thread
// for the logits, a column a thread for the sum over the rows; running maximum and sum.
// ---------------------------------------------------------------------------------------------
struct PackedDev {
  const DState* ds;
  const uint16_t* q;
  float* out;
  int64_t q_stride, out_stride;
  int layer;
  float qscale;  // scale * log2(e)
};

template <typename T, int D>
__global__ void __launch_bounds__(128) packed_decode_kernel(Geometry g, Static st, PackedBuffers pb, PackedDev p) {
  using R = PackedRow<D>;
  __shared__ float qs[D], raw[D], ps[128], red[4], gsum[R::G];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.x % g.H, s = (blockIdx.x / g.H) % g.b, li = blockIdx.x / (g.H * g.b);
  const DState ds = p.ds[s];
  if (ds.len <= ds.begin) return;
  const uint16_t* q = p.q + li * p.q_stride + ((int64_t)s * g.H + h) * D;
  if (tid < D) raw[tid] = T::f1(q[tid]);
  __syncthreads();
  if (tid < D) {
    float x = raw[tid];
    if (tid < g.rot) {
      const int half = g.rot / 2;
      float sn, cs;
      rope_sincos_full(ds.qpos, st.rope_g[tid < half ? tid : tid - half], &sn, &cs);
      x = tid < half ? x * cs - raw[tid + half] * sn : x * cs + raw[tid - half] * sn;
    }
    qs[tid] = x;
  }
  __syncthreads();
  if (tid < R::G) {
    float x = 0.f;
    for (int c = 32 * tid; c < min(D, 32 * tid + 32); ++c) x += qs[c];
    gsum[tid] = x;
  }
  const int64_t row0 = (int64_t)(p.layer + li) * g.H * g.C + st.seq_row0[s] + (int64_t)h * st.cap[s];
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int r0 = ds.begin; r0 < ds.len; r0 += 128) {
    const int r = r0 + tid, n = min(128, ds.len - r0);
    const bool seen = r < ds.len && !(r >= ds.mask_lo && r < ds.mask_hi);
    __syncthreads();
    float z = -INFINITY;
    if (seen) {
      z = 0.f;
      for (int gg = 0; gg < R::G; ++gg) {
        float x = 0.f;
        for (int w = 4 * gg; w < min(R::W, 4 * gg + 4); ++w) {
          const uint32_t word = reinterpret_cast<const uint32_t*>(pb.kc)[(row0 + r) * R::W + w];
          for (int e = 0; e < 8; ++e) x = fmaf(qs[8 * w + e], (float)(word >> (4 * e) & 15u), x);
        }
        const uint32_t pair = pb.kp[(row0 + r) * R::G + gg];
        z += T::f1((uint16_t)pair) * x + T::f1((uint16_t)(pair >> 16)) * gsum[gg];
      }
      z *= p.qscale;
    }
    float mx = z;
    for (int i = 16; i > 0; i >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, i));
    if (lane == 0) red[warp] = mx;
    __syncthreads();
    mx = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    const float ref = mx == -INFINITY ? 0.f : mx;
    ps[tid] = seen ? exp2f(z - ref) : 0.f;
    const float f = exp2f(m - ref);
    __syncthreads();
    m = mx;
    l *= f;
    o *= f;
    for (int i = 0; i < n; ++i) {
      if (r0 + i >= ds.mask_lo && r0 + i < ds.mask_hi) continue;
      l += ps[i];
      if (tid < D) {
        const uint32_t word = reinterpret_cast<const uint32_t*>(pb.vc)[(row0 + r0 + i) * R::W + tid / 8];
        const uint32_t pair = pb.vp[(row0 + r0 + i) * R::G + tid / 32];
        o += ps[i] * fmaf(T::f1((uint16_t)pair), (float)(word >> (4 * (tid % 8)) & 15u), T::f1((uint16_t)(pair >> 16)));
      }
    }
  }
  if (tid < D) p.out[li * p.out_stride + ((int64_t)s * g.H + h) * D + tid] = o / l;
}

template <typename F>
cudaError_t by_type(const Geometry& g, F&& f) {
  auto dtype = [&](auto dc) { return g.dtype == 1 ? f(BF16T{}, dc) : f(F16T{}, dc); };
  switch (g.D) {
    case 64:
      return dtype(std::integral_constant<int, 64>{});
    case 80:
      return dtype(std::integral_constant<int, 80>{});
    case 96:
      return dtype(std::integral_constant<int, 96>{});
    case 128:
      return dtype(std::integral_constant<int, 128>{});
    default:
      return cudaErrorInvalidValue;
  }
}

}  // namespace

cudaError_t launch_packed_append(const Geometry& g, const Static& st, const Buffers& buf, const PackedBuffers& pb,
                                 const TokPlan* plan, const AppendImage* img, size_t img_bytes, size_t plan_off, void* dyn,
                                 int64_t n_plan, int64_t n_in, int m0, int n_layers, bool write_meta, const void* k_in,
                                 const void* v_in, cudaStream_t stream) {
  return by_type(g, [&](auto t, auto dc) {
    using T = decltype(t);
    constexpr int D = decltype(dc)::value;
    const uint16_t *k = static_cast<const uint16_t*>(k_in), *v = static_cast<const uint16_t*>(v_in);
    // one token a sequence: neighbours in the plan are rows of different streams
    const int tg = n_plan >= kPackTokens * (int64_t)g.b ? kPackTokens : 1;
    const unsigned blocks = (unsigned)std::min<int64_t>((n_plan + tg - 1) / tg * n_layers, 16384);
    if (img)
      packed_append_image_kernel<T, D><<<blocks, kPackThreads, 0, stream>>>(g, st, buf, pb, *img, (int)img_bytes, (int)plan_off,
                                                                           static_cast<uint4*>(dyn), n_plan, n_in, n_layers,
                                                                           tg, k, v);
    else
      packed_append_kernel<T, D><<<blocks, kPackThreads, 0, stream>>>(g, st, buf, pb, plan, n_plan, n_in, m0, n_layers, tg,
                                                                     write_meta, k, v);
    return cudaGetLastError();
  });
}

cudaError_t launch_packed_move(const Geometry& g, const Static& st, const PackedBuffers& pb, const AffSeq* aff, int n_aff,
                               const int32_t* src_map, cudaStream_t stream) {
  return by_type(g, [&](auto, auto dc) {
    packed_move_kernel<decltype(dc)::value>
        <<<(unsigned)((int64_t)n_aff * g.M * 2 * g.H), kMoveThreads, 0, stream>>>(g, st, pb, aff, src_map);
    return cudaGetLastError();
  });
}

cudaError_t launch_packed_decode(const Geometry& g, const Static& st, const PackedBuffers& pb, const DecodeArgs& a,
                                 int* status, int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan) {
  (void)status;
  (void)num_sms;
  PackedDev p;
  p.ds = a.dstate;
  p.q = static_cast<const uint16_t*>(a.q);
  p.out = a.out;
  p.q_stride = a.q_layer_stride;
  p.out_stride = a.out_layer_stride;
  p.layer = a.layer;
  p.qscale = a.scale * 1.4426950408889634f;
  const int64_t blocks = (int64_t)a.n_layers * g.b * g.H;
  *grid = (int)blocks;
  *plan = {5, (int)blocks * 4, 128, 1};
  return by_type(g, [&](auto t, auto dc) {
    packed_decode_kernel<decltype(t), decltype(dc)::value><<<(unsigned)blocks, 128, 0, stream>>>(g, st, pb, p);
    return cudaGetLastError();
  });
}

}  // namespace kvc
