// Kernels of a cache whose rows are held in 4 bits (packed.cuh has the format).
//
//   packed_append_kernel  new tokens' K/V rows, K rotated and rounded as the 16-bit append does it, into codes and pairs
//   packed_move_kernel    the row moves of a compaction
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "kernels.hpp"
#include "packed.cuh"
#include "turned_keys.cuh"

namespace kvc {
namespace {

// ---------------------------------------------------------------------------------------------
// Append
// ---------------------------------------------------------------------------------------------
// A block takes (layer, group of TG tokens) units.  A lane takes a group of columns of a row (the step and its reciprocal once
// for 32 columns), except of keys that are rotated: there eight columns, whose group's four lanes are side by side.  The
// tokens of a unit come before the heads, so that a warp writes the rows of neighbouring tokens, which are neighbours in a
// stream, together.  Memory and the load's way bound it: 2,000 tokens of 8 layers of 32 heads of 128 columns take 65 us with
// the call (floor 52; eight columns a lane throughout: 128).
constexpr int kPackThreads = 256;
constexpr int kPackTokens = 8;

template <typename T, int D>
__device__ __forceinline__ void pack_units(const Geometry& g, const Static& st, const Buffers& buf, const PackedBuffers& pb,
                                           const TokPlan* plan, int64_t ntok, int64_t n_in, int m0, int n_layers, int tg,
                                           int write_meta, const uint16_t* __restrict__ k_in,
                                           const uint16_t* __restrict__ v_in) {
  using R = PackedRow<D>;
  // A decode's workers may start: they wait for this kernel before they read anything or let what follows them start.
  pdl_launch_dependents();
  __shared__ float2 rope_cs[kPackTokens][D / 2];  // (cos, sin) of the tokens' rotated pairs
  const int H = g.H, half = g.rot / 2;
  const int64_t groups = (ntok + tg - 1) / tg, n_units = groups * n_layers;
  const int tsh = tg == 1 ? 0 : 3;
  static_assert(kPackTokens == 8);
  // rows of a lane a group: the values, and the keys that are not rotated
  const int n_groups = (half > 0 ? H : 2 * H) * tg * R::G, n_items = half > 0 ? H * tg * R::CP : 0;
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
    auto source = [&](const uint16_t* in, const TokPlan& tp, int h) {
      return in + (((int64_t)l * n_in + tp.in_tok) * H + h) * D;
    };
    auto target = [&](const TokPlan& tp, int h) {
      return (int64_t)(m0 + l) * H * g.C + st.seq_row0[tp.s] + (int64_t)h * st.cap[tp.s] + tp.row;
    };
    for (int i = threadIdx.x; i < n_groups; i += blockDim.x) {
      const int gi = i % R::G, j = i / R::G, t = j & (tg - 1), hv = j >> tsh;
      if (t >= nt) continue;
      const bool is_v = hv < H;
      const int h = is_v ? hv : hv - H;
      const TokPlan tp = plan[t0 + t];
      uint32_t code[4];
      const uint32_t pair = pack_group<T, D>(source(is_v ? v_in : k_in, tp, h), gi, code);
      store_group<D>(is_v ? pb.vc : pb.kc, is_v ? pb.vp : pb.kp, target(tp, h), gi, code, pair);
    }
    // a multiple of 32 for every warp: the lanes of a group reduce together
    for (int i = threadIdx.x; i < (n_items + 31) / 32 * 32; i += blockDim.x) {
      const int c = i % R::CP, j = i / R::CP, t = j & (tg - 1), h = j >> tsh;
      const bool active = h < H && t < nt && c < R::W;
      const TokPlan tp = plan[t0 + min(t, nt - 1)];
      uint32_t x[4] = {0, 0, 0, 0};
      if (active) {
        const uint16_t* src = source(k_in, tp, h);
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(src + 8 * c));
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
        if (8 * c < g.rot) {
          const bool first = 8 * c < half;
          const int p0 = first ? 8 * c : 8 * c - half;
          const uint4 b = __ldg(reinterpret_cast<const uint4*>(src + (first ? 8 * c + half : p0)));
          const uint32_t bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = T::f2(x[e]), o = T::f2(bv[e]);
            const float2 r0 = rope_cs[t][p0 + 2 * e], r1 = rope_cs[t][p0 + 2 * e + 1];
            x[e] = first ? T::r2(turned_first(f.x, o.x, r0), turned_first(f.y, o.y, r1))
                         : T::r2(turned_second(o.x, f.x, r0), turned_second(o.y, f.y, r1));
          }
        }
      }
      uint32_t pair;
      const uint32_t word = pack8<T>(x, active, &pair);
      if (!active) continue;
      const int64_t row = target(tp, h);
      reinterpret_cast<uint32_t*>(pb.kc)[row * R::W + c] = word;
      if (c % 4 == 0) pb.kp[row * R::G + c / 4] = pair;
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
    packed_move_kernel(Geometry g, Static st, PackedBuffers pb, const AffSeq* __restrict__ aff,
                       const int32_t* __restrict__ src_map) {
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

}  // namespace kvc
