// The decode over a cache whose rows are held in 4 bits (packed.cuh has the format).
//
//   out = sum_j softmax_j(scale <q, k_j>) v_j,  k_j = lo + step c_j a group of 32 columns (v_j likewise), c_j from 0 to 15:
//   <q, k_j> = sum over the groups of step <q, c_j - 8> + (lo + 8 step) sum(q),
//   sum_j p_j v_j = sum_j (p_j step) (c_j - 8) + sum_j p_j (lo + 8 step).
//
// (Around 8, because sums of codes would be far larger than what is left of them: with c_j itself the outputs of 1,024 rows
// were off by some ten times as much.)
//
// Both sums of products go through 16 x 8 x 16 matrix instructions, whose other operand has eight columns: the query's
// columns of each group apart (zero elsewhere), and the weights times each group's steps, each as two f16 parts (22 bits
// of a value) in columns 2 g and 2 g + 1.  One query a head leaves the arithmetic small but the unpacking large: a 64-column
// row is 64 codes, and at the memory's rate an SM has 3 lane-instructions for each.  As matrix operands two codes need two and
// a quarter: masked out of the word into the mantissa of two f16 numbers of 1,024 and up, and those brought down to
// code - 8 by a packed sum, or a packed fused product and sum for a code four bits up.  (Codes as subnormal f16 numbers need
// one, but the matrix unit aligns its products by the exponents, as if their leading bits were set: 1.1e-5 of the norm off.)
//
// The work: the tiles of 64 rows of all (layer, sequence, head) segments in a row, an equal share for each warp that fits the
// GPU.  A warp is a worker of its own, with a ring of stages in shared memory that 1-D bulk copies fill (codes and pairs of
// K and V, four copies a tile).  A segment that spans several workers is joined by the last of them to finish, from parts in
// the workspace, in the workers' order.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "kernels.hpp"
#include "packed.cuh"

namespace kvc {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kTile = kPackedTile;

template <int D, int S_>
struct Shape {
  using R = PackedRow<D>;
  static constexpr int S = S_;
  static constexpr int KC = kTile * R::RB, KP = kTile * R::PB;
  static constexpr int STAGE = 2 * (KC + KP);  // K codes, K pairs, V codes, V pairs
  static constexpr int PS = 2 * 8 * 32 * 2;    // weights times steps: [32-row block][column][row] f16; the query between pieces
  static constexpr int SMEM = S * STAGE + PS + 8 * S;
  static_assert(4 * D <= PS);
};

struct PackedDev {
  const DState* ds;
  const int64_t* P;  // prefix sums of the sequences' tiles
  int64_t R;         // tiles of a layer
  int n_layers, layer;
  int NW;
  const uint16_t* q;
  float* out;
  int64_t q_stride, out_stride;
  float* parts;   // [NW][2][D + 4]: maximum, sum, two unused, columns
  int* counters;  // [NW], zero between launches
  int* status;
  float qscale;   // scale * log2(e)
  unsigned long long limit_ns;
  int kv_before_wait;
};

// A tile among all: x-th of the launch, r-th of its segment's Lc.
struct Cursor {
  int64_t x, Lc, r;
  int s, h, layer;
  // to the next tile, which exists if x + 1 < hi
  __device__ __forceinline__ void advance(int64_t hi, const int64_t* P, int H, int b) {
    ++x;
    if (++r < Lc || x >= hi) return;
    r = 0;
    if (++h == H) {
      h = 0;
      do {
        if (++s == b) {
          s = 0;
          ++layer;
        }
      } while (P[s + 1] == P[s]);
      Lc = P[s + 1] - P[s];
    }
  }
};

// The worker whose share [w Rt / NW, (w + 1) Rt / NW) holds tile x.
__device__ __forceinline__ int worker_of(int64_t x, int64_t Rt, int NW) { return (int)(((x + 1) * NW - 1) / Rt); }

// The sequence that holds tile o of a layer: the last s with H P[s] <= o, a search of the whole warp.
__device__ __forceinline__ int seq_of(const int64_t* P, int b, int H, int64_t o, int lane) {
  int a = 0, z = b;
  while (z - a > 1) {
    const int step = (z - a + 31) / 32, k = a + lane * step;
    const unsigned bal = __ballot_sync(kFull, k < z && (int64_t)H * P[k] <= o);
    a += (31 - __clz(bal)) * step;
    z = min(z, a + step);
  }
  return a;
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two codes of a word as f16 numbers less 8: those in bits 0 to 3 of each half, or in bits 4 to 7.
__device__ __forceinline__ uint32_t low_codes(uint32_t w) {
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(x) : "r"(w));  // 1024 + c
  const __half2 h = __hadd2(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half(0xE408)));  // - 1032
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t high_codes(uint32_t w) {
  uint32_t x;
  asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(x) : "r"(w));  // 1024 + 16 c
  const __half2 h = __hfma2(*reinterpret_cast<const __half2*>(&x), __half2half2(__ushort_as_half(0x2C00)),   // 1 / 16
                            __half2half2(__ushort_as_half(0xD480)));                                          // - 72
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ float half_bits(uint32_t h) { return __half2float(__ushort_as_half((uint16_t)h)); }
__device__ __forceinline__ uint32_t pack_halves(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Two steps of 16 columns of the keys' product, from one code word of row g (a) and of row g + 8 (b) each.
__device__ __forceinline__ void key_word(float (&c)[4], uint32_t a, uint32_t b, const uint32_t (&q)[4]) {
  mma(c, low_codes(a), low_codes(b), high_codes(a), high_codes(b), q[0], q[1]);
  a >>= 8;
  b >>= 8;
  mma(c, low_codes(a), low_codes(b), high_codes(a), high_codes(b), q[2], q[3]);
}

// 16 rows of the values' product for four columns: two of rows 0, 4 (x01) and 8, 12 (x23), and the two eight bits up.
__device__ __forceinline__ void value_pair(float (&c)[4], uint32_t x01, uint32_t x23, uint32_t b0, uint32_t b1) {
  mma(c, low_codes(x01), high_codes(x01), low_codes(x23), high_codes(x23), b0, b1);
}

template <typename T, int D, int S>
__global__ void __launch_bounds__(32, D == 128 ? 10 : D == 96 ? 13 : 16)
    packed_decode_kernel(Geometry g, Static st, PackedBuffers pb, PackedDev p) {
  using C = Shape<D, S>;
  using R = PackedRow<D>;
  constexpr int G = R::G;
  constexpr int KW = D == 128 ? 4 : 2;              // code words of a row a lane has of the keys
  constexpr int NT = D / 16;                        // tiles of 16 columns of the values
  constexpr int QF = 2 * (D / 16);                  // registers of the query
  extern __shared__ __align__(128) unsigned char smem[];
  pdl_launch_dependents();
  const int lane = threadIdx.x, gr = lane >> 2, t = lane & 3;
  const int wid = blockIdx.x, H = g.H;
  const int64_t Rt = (int64_t)p.n_layers * p.R;
  const int64_t lo = (int64_t)wid * Rt / p.NW, hi = (int64_t)(wid + 1) * Rt / p.NW;

  unsigned char* ps = smem + S * C::STAGE;
  float* qs = reinterpret_cast<float*>(ps);
  uint64_t* full = reinterpret_cast<uint64_t*>(ps + C::PS);
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < S; ++i) mbar_init(&full[i], 1);
    fence_mbar_init();
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (!p.kv_before_wait) pdl_wait();

  Cursor ci;  // consumed tiles
  ci.x = lo;
  ci.layer = (int)(lo / p.R);
  {
    const int64_t o = lo - (int64_t)ci.layer * p.R;
    ci.s = seq_of(p.P, g.b, H, o, lane);
    const int64_t P0 = p.P[ci.s];
    ci.Lc = p.P[ci.s + 1] - P0;
    ci.h = (int)((o - (int64_t)H * P0) / ci.Lc);
    ci.r = o - (int64_t)H * P0 - (int64_t)ci.h * ci.Lc;
  }
  Cursor ii = ci;  // issued tiles (lane 0)
  int is = -1, i_begin = 0, i_len = 0, i_cap = 0;
  int64_t i_row0 = 0;
  auto issue = [&](int stage) {
    if (ii.s != is) {
      is = ii.s;
      const DState d = p.ds[is];
      i_begin = d.begin / kPackedRows * kPackedRows;
      i_len = d.len;
      i_row0 = st.seq_row0[is];
      i_cap = st.cap[is];
    }
    const int r0 = i_begin + (int)ii.r * kTile;
    const uint32_t n = (uint32_t)((min(kTile, i_len - r0) + kPackedRows - 1) / kPackedRows * kPackedRows);
    const int64_t row = (int64_t)(p.layer + ii.layer) * H * g.C + i_row0 + (int64_t)ii.h * i_cap + r0;
    unsigned char* to = smem + stage * C::STAGE;
    mbar_arrive_expect_tx(&full[stage], 2 * n * (R::RB + R::PB));
    bulk_g2s(to, pb.kc + row * R::RB, n * R::RB, &full[stage]);
    bulk_g2s(to + C::KC, pb.kp + row * R::G, n * R::PB, &full[stage]);
    bulk_g2s(to + C::KC + C::KP, pb.vc + row * R::RB, n * R::RB, &full[stage]);
    bulk_g2s(to + 2 * C::KC + C::KP, pb.vp + row * R::G, n * R::PB, &full[stage]);
    ii.advance(hi, p.P, H, g.b);
  };
  // a decode before this one writes neither rows nor state: they may come before it is complete, while the query, the outputs
  // and the parts may be shared with it
  if (lane == 0)
    for (int i = 0; i < S && ii.x < hi; ++i) issue(i);
  if (p.kv_before_wait) pdl_wait();

  // the query of a segment, fetched a piece ahead: columns lane + 32 j, and those they are rotated with
  constexpr int QL = (D + 31) / 32;
  float qa[QL], qb[QL];
  auto fetch_q = [&](const Cursor& c) {
    const uint16_t* row = p.q + (int64_t)c.layer * p.q_stride + ((int64_t)c.s * H + c.h) * D;
    const int half = g.rot / 2;
#pragma unroll
    for (int j = 0; j < QL; ++j) {
      const int k = lane + 32 * j;
      qa[j] = qb[j] = 0.f;
      if (k < D) {
        qa[j] = T::f1(row[k]);
        if (k < g.rot) qb[j] = T::f1(row[k < half ? k + half : k - half]);
      }
    }
  };
  fetch_q(ci);

  uint32_t qf[QF];      // the query as the keys' other operand
  float qsum = 0.f;     // its sum over group t's columns, times qscale
  float kscale = 0.f;   // of a product of codes and the query's parts
  float o[2 * NT], l = 0.f, los[G], m = -INFINITY;
  DState ds = p.ds[ci.s];
  int stage = 0;
  uint32_t phase = 0;
  bool fresh = true;

  while (ci.x < hi) {
    if (fresh) {  // a new piece
      fresh = false;
      float sum[QL], big = 0.f;
#pragma unroll
      for (int j = 0; j < QL; ++j) {
        const int k = lane + 32 * j;
        if (k < g.rot) {
          const int half = g.rot / 2;
          float sn, cs;
          rope_sincos_full(ds.qpos, st.rope_g[k < half ? k : k - half], &sn, &cs);
          qa[j] = k < half ? qa[j] * cs - qb[j] * sn : qa[j] * cs + qb[j] * sn;
        }
        sum[j] = qa[j];
        big = fmaxf(big, fabsf(qa[j]));
      }
#pragma unroll
      for (int i = 16; i > 0; i >>= 1) {
        big = fmaxf(big, __shfl_xor_sync(kFull, big, i));
#pragma unroll
        for (int j = 0; j < QL; ++j) sum[j] += __shfl_xor_sync(kFull, sum[j], i);
      }
      // the largest column goes to [2^13, 2^14): it and a second part are then far from f16's ends
      const int e = big > 0.f && big < INFINITY ? max(-115, min(115, 13 - (int)(__float_as_uint(big) >> 23) + 127)) : 0;
      const float up = __uint_as_float((uint32_t)(127 + e) << 23);
      kscale = p.qscale * __uint_as_float((uint32_t)(127 - e) << 23);
      qsum = (t == 0 ? sum[0] : t == 1 ? sum[1] : t == 2 && QL > 2 ? sum[QL > 2 ? 2 : 0] : QL > 3 ? sum[QL > 3 ? 3 : 0] : 0.f) * p.qscale;
      __syncwarp();  // the weights of the piece before are read
#pragma unroll
      for (int j = 0; j < QL; ++j)
        if (lane + 32 * j < D) qs[lane + 32 * j] = qa[j] * up;
      __syncwarp();
      // column gr of the operand: group gr / 2, part gr % 2
      auto part = [&](int k) {
        const float x = (k >> 5) == (gr >> 1) ? qs[k] : 0.f;
        const float h = __half2float(__float2half_rn(x));
        return gr & 1 ? x - h : h;
      };
      auto word = [&](int k, uint32_t* f) {
        f[0] = pack_halves(part(k), part(k + 4));
        f[1] = pack_halves(part(k + 1), part(k + 5));
        f[2] = pack_halves(part(k + 2), part(k + 6));
        f[3] = pack_halves(part(k + 3), part(k + 7));
      };
#pragma unroll
      for (int i = 0; i < KW; ++i) word(8 * (KW * t + i), qf + 4 * i);
      if constexpr (D == 96) word(64 + 8 * t, qf + 8);
      if constexpr (D == 80) {
        qf[8] = pack_halves(part(64 + 4 * t), part(64 + 4 * t + 2));
        qf[9] = pack_halves(part(64 + 4 * t + 1), part(64 + 4 * t + 3));
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) o[i] = 0.f;
#pragma unroll
      for (int i = 0; i < G; ++i) los[i] = 0.f;
      l = 0.f;
      m = -INFINITY;
    }

    // ---- a tile
    if (!__all_sync(kFull, mbar_wait_bounded(&full[stage], phase, p.limit_ns))) {
      if (lane == 0) {
        atomicOr(p.status, STATUS_TIMEOUT);
        // the copies that are still in flight end before their memory does
        for (int64_t i = ci.x; i < ii.x; ++i) {
          mbar_wait_bounded(&full[stage], phase, p.limit_ns);
          if (++stage == S) {
            stage = 0;
            phase ^= 1;
          }
        }
      }
      __syncwarp();
      return;  // the segment is not joined
    }
    const unsigned char* kc = smem + stage * C::STAGE;
    const uint32_t* kp = reinterpret_cast<const uint32_t*>(kc + C::KC);
    const unsigned char* vc = kc + C::KC + C::KP;
    const uint32_t* vp = reinterpret_cast<const uint32_t*>(vc + C::KC);
    const int r0 = ds.begin / kPackedRows * kPackedRows + (int)ci.r * kTile;
    const int nb = ds.len - r0 > 32 ? 2 : 1;  // blocks of 32 rows with rows

    float z[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      z[b] = 0.f;
      if (b < nb) {
        float v[4];  // lane t's group's part of the logits of rows gr + 8 i
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int row = 32 * b + 16 * a + gr;
          const unsigned char *x = kc + row * R::RB, *y = x + 8 * R::RB;
          float c[4] = {0.f, 0.f, 0.f, 0.f};
          if constexpr (D == 128) {
            const uint4 u = *reinterpret_cast<const uint4*>(x + 16 * t), w = *reinterpret_cast<const uint4*>(y + 16 * t);
            key_word(c, u.x, w.x, reinterpret_cast<const uint32_t(&)[4]>(qf[0]));
            key_word(c, u.y, w.y, reinterpret_cast<const uint32_t(&)[4]>(qf[4]));
            key_word(c, u.z, w.z, reinterpret_cast<const uint32_t(&)[4]>(qf[8]));
            key_word(c, u.w, w.w, reinterpret_cast<const uint32_t(&)[4]>(qf[12]));
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(x + 8 * t), w = *reinterpret_cast<const uint2*>(y + 8 * t);
            key_word(c, u.x, w.x, reinterpret_cast<const uint32_t(&)[4]>(qf[0]));
            key_word(c, u.y, w.y, reinterpret_cast<const uint32_t(&)[4]>(qf[4]));
          }
          if constexpr (D == 96)
            key_word(c, *reinterpret_cast<const uint32_t*>(x + 32 + 4 * t), *reinterpret_cast<const uint32_t*>(y + 32 + 4 * t),
                     reinterpret_cast<const uint32_t(&)[4]>(qf[8]));
          if constexpr (D == 80) {  // four columns: the second byte's go to the upper half
            const uint32_t u = __byte_perm(*reinterpret_cast<const uint16_t*>(x + 32 + 2 * t), 0, 0x4140);
            const uint32_t w = __byte_perm(*reinterpret_cast<const uint16_t*>(y + 32 + 2 * t), 0, 0x4140);
            mma(c, low_codes(u), low_codes(w), high_codes(u), high_codes(w), qf[8], qf[9]);
          }
          v[2 * a] = v[2 * a + 1] = 0.f;
          if (t < G) {
            const uint32_t p0 = kp[row * G + t], p1 = kp[(row + 8) * G + t];
            const float s0 = T::f1((uint16_t)p0), s1 = T::f1((uint16_t)p1);
            v[2 * a] = fmaf(s0, (c[0] + c[1]) * kscale, fmaf(8.f, s0, T::f1((uint16_t)(p0 >> 16))) * qsum);
            v[2 * a + 1] = fmaf(s1, (c[2] + c[3]) * kscale, fmaf(8.f, s1, T::f1((uint16_t)(p1 >> 16))) * qsum);
          }
        }
        // the sum over the groups; lane t is left with row gr + 8 t
        const bool odd = t & 1, two = t & 2;
        const float s0 = (odd ? v[1] : v[0]) + __shfl_xor_sync(kFull, odd ? v[0] : v[1], 1);
        const float s1 = (odd ? v[3] : v[2]) + __shfl_xor_sync(kFull, odd ? v[2] : v[3], 1);
        z[b] = (two ? s1 : s0) + __shfl_xor_sync(kFull, two ? s0 : s1, 2);
      }
    }

    // the lane's rows (gr + 8 t of each block): the values' pairs, and the exponent of the row's largest step, which goes
    // into the running maximum, so that weight times step stays in f16's range whatever the steps are
    bool seen[2];
    uint32_t vpair[2][G];
    float zs[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int row = 32 * b + 8 * t + gr, at = r0 + row;
      seen[b] = at >= ds.begin && at < ds.len && !(at >= ds.mask_lo && at < ds.mask_hi);
      uint32_t big = 0;
#pragma unroll
      for (int i = 0; i < G; ++i) {
        vpair[b][i] = vp[row * G + i];
        const uint32_t s = vpair[b][i] & 0xFFFFu;
        if (s < (std::is_same_v<T, F16T> ? 0x7C00u : 0x7F80u)) big = max(big, s);
        if constexpr (std::is_same_v<T, BF16T>) {  // and of 2^-20 of its least values, which f32 would not hold times a weight
          const uint32_t x = vpair[b][i] >> 16 & 0x7FFFu;
          if (x < 0x7F80u) big = max(big, x > (20u << 7) ? x - (20u << 7) : 0u);
        }
      }
      // from 2^-88 on: a weight is at most 2^102, and the sum of 2^25 of them in f32's range (with smaller steps the weights times
      // them end earlier than 2^15, and below 2^-110 they lose bits)
      const int e = max((int)(__float_as_uint(T::f1((uint16_t)big)) >> 23) - 127, -88);
      zs[b] = seen[b] ? z[b] + (float)e : -INFINITY;
    }
    float mx = fmaxf(zs[0], zs[1]);
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, i));
    if (mx > m + 4.f) {  // of the warp: the reference moves where weights times steps would pass 2^15
      const float f = exp2f(m - mx);
#pragma unroll
      for (int i = 0; i < 2 * NT; ++i) o[i] *= f;
#pragma unroll
      for (int i = 0; i < G; ++i) los[i] *= f;
      l *= f;
      m = mx;
    }
    const float ref = m == -INFINITY ? 10.f : 10.f - m;
    uint16_t* pw = reinterpret_cast<uint16_t*>(ps);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float w = seen[b] ? exp2f(z[b] + ref) : 0.f;
      l += w;
      const int at = 256 * b + 8 * (gr & 3) + 2 * t + (gr >> 2);  // of row r = gr + 8 t: 8 (r % 4) + r / 4
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const float step = T::f1((uint16_t)vpair[b][i]), least = T::f1((uint16_t)(vpair[b][i] >> 16));
        const float x = seen[b] ? w * step : 0.f;
        if (seen[b]) los[i] = fmaf(w, fmaf(8.f, step, least), los[i]);
        const __half h = __float2half_rn(x);
        pw[at + 64 * i] = __half_as_ushort(h);
        pw[at + 64 * i + 32] = __half_as_ushort(__float2half_rn(x - __half2float(h)));
      }
    }
    __syncwarp();

    float acc[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if (b < nb) {
        const uint4 wb = *reinterpret_cast<const uint4*>(pw + 256 * b + 32 * gr + 8 * t);
#pragma unroll
        for (int k = 0; k < 2; ++k) {  // 16 rows: t + 4 i of the block's half
          const uint32_t b0 = k ? wb.z : wb.x, b1 = k ? wb.w : wb.y;
          const unsigned char* x = vc + (32 * b + 16 * k + t) * R::RB;
          auto word = [&](int i, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
            uint32_t u = __byte_perm(w0, w1, 0x5410), v = __byte_perm(w2, w3, 0x5410);
            value_pair(acc[i], u, v, b0, b1);
            value_pair(acc[i + 1], u >> 8, v >> 8, b0, b1);
            u = __byte_perm(w0, w1, 0x7632), v = __byte_perm(w2, w3, 0x7632);
            value_pair(acc[i + 2], u, v, b0, b1);
            value_pair(acc[i + 3], u >> 8, v >> 8, b0, b1);
          };
          if constexpr (D == 128) {
            const uint2 w0 = *reinterpret_cast<const uint2*>(x + 8 * gr);
            const uint2 w1 = *reinterpret_cast<const uint2*>(x + 4 * R::RB + 8 * gr);
            const uint2 w2 = *reinterpret_cast<const uint2*>(x + 8 * R::RB + 8 * gr);
            const uint2 w3 = *reinterpret_cast<const uint2*>(x + 12 * R::RB + 8 * gr);
            word(0, w0.x, w1.x, w2.x, w3.x);
            word(4, w0.y, w1.y, w2.y, w3.y);
          } else {
            auto at = [&](int i) { return *reinterpret_cast<const uint32_t*>(x + 4 * i * R::RB + 4 * gr); };
            word(0, at(0), at(1), at(2), at(3));
          }
          if constexpr (D == 96) {  // the last four words, half a word a lane
            auto at = [&](int i) { return (uint32_t)*reinterpret_cast<const uint16_t*>(x + 4 * i * R::RB + 32 + 2 * gr); };
            const uint32_t u = __byte_perm(at(0), at(1), 0x5410), v = __byte_perm(at(2), at(3), 0x5410);
            value_pair(acc[4], u, v, b0, b1);
            value_pair(acc[5], u >> 8, v >> 8, b0, b1);
          }
          if constexpr (D == 80) {  // the last two, a byte a lane
            auto at = [&](int i) { return (uint32_t)x[4 * i * R::RB + 32 + gr]; };
            value_pair(acc[4], at(0) | at(1) << 16, at(2) | at(3) << 16, b0, b1);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      o[2 * i] += acc[i][0] + acc[i][1];
      o[2 * i + 1] += acc[i][2] + acc[i][3];
    }
    __syncwarp();  // the stage and the weights are read
    if (lane == 0 && ii.x < hi) issue(stage);
    if (++stage == S) {
      stage = 0;
      phase ^= 1;
    }

    // ---- the end of a piece
    const Cursor was = ci;
    ci.advance(hi, p.P, H, g.b);
    if (ci.x < hi && was.r + 1 < was.Lc) continue;
    if (ci.x < hi) fetch_q(ci);
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) {
      l += __shfl_xor_sync(kFull, l, i);
#pragma unroll
      for (int k = 0; k < G; ++k) los[k] += __shfl_xor_sync(kFull, los[k], i);
    }
    // lane (gr, t) has the columns of its words for group t: o[2 i], o[2 i + 1] are columns col(i), col(i) + 1
    auto col = [&](int i) {
      if (D == 128) return 16 * gr + 8 * (i / 4) + 2 * (i % 4);
      return i < 4 ? 8 * gr + 2 * i : D == 96 ? 64 + 4 * gr + 2 * (i - 4) : 64 + 2 * gr;
    };
    float mine = los[0];  // group t's
#pragma unroll
    for (int k = 1; k < G; ++k)
      if (t == k) mine = los[k];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      o[2 * i] += mine;
      o[2 * i + 1] += mine;
    }
    const int64_t seg0 = ci.x - (was.r + 1), seg1 = seg0 + was.Lc;  // the segment's tiles among all
    float* orow = p.out + (int64_t)was.layer * p.out_stride + ((int64_t)was.s * H + was.h) * D;
    if (seg0 >= lo && seg1 <= hi) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
        if (t == col(i) / 32) {
          orow[col(i)] = o[2 * i] / l;
          orow[col(i) + 1] = o[2 * i + 1] / l;
        }
    } else {
      // a worker has at most two parts: of a segment that began before it, and of one that goes on behind it
      float* part = p.parts + ((int64_t)wid * 2 + (seg0 < lo ? 0 : 1)) * (D + 4);
#pragma unroll
      for (int i = 0; i < NT; ++i)
        if (t == col(i) / 32) {
          __stcg(part + 4 + col(i), o[2 * i]);
          __stcg(part + 5 + col(i), o[2 * i + 1]);
        }
      if (lane == 0) {
        __stcg(part, m);
        __stcg(part + 1, l);
      }
      const int first = worker_of(seg0, Rt, p.NW), last = worker_of(seg1 - 1, Rt, p.NW);
      __threadfence();
      __syncwarp();
      int done = 0;
      if (lane == 0) done = atomicAdd(p.counters + first, 1) == last - first;
      if (__shfl_sync(kFull, done, 0)) {
        __threadfence();
        auto at = [&](int w) { return p.parts + ((int64_t)w * 2 + (w == first ? 1 : 0)) * (D + 4); };
        float big = -INFINITY;
        for (int w = first + lane; w <= last; w += 32) big = fmaxf(big, __ldcg(at(w)));
#pragma unroll
        for (int i = 16; i > 0; i >>= 1) big = fmaxf(big, __shfl_xor_sync(kFull, big, i));
        float sum = 0.f, x[QL];
#pragma unroll
        for (int j = 0; j < QL; ++j) x[j] = 0.f;
        for (int w = first; w <= last; ++w) {
          const float* a = at(w);
          const float mw = __ldcg(a);
          const float f = mw == -INFINITY ? 0.f : exp2f(mw - big);
          sum = fmaf(f, __ldcg(a + 1), sum);
#pragma unroll
          for (int j = 0; j < QL; ++j)
            if (lane + 32 * j < D) x[j] = fmaf(f, __ldcg(a + 4 + lane + 32 * j), x[j]);
        }
#pragma unroll
        for (int j = 0; j < QL; ++j)
          if (lane + 32 * j < D) orow[lane + 32 * j] = x[j] / sum;
        if (lane == 0) p.counters[first] = 0;
      }
    }
    fresh = true;
    if (ci.x < hi && ci.s != was.s) ds = p.ds[ci.s];
  }
}

template <int D>
constexpr int kStages = 2;

template <typename T, int D, int S>
cudaError_t launch_t(const Geometry& g, const Static& st, const PackedBuffers& pb, PackedDev p, int device, int num_sms,
                     cudaStream_t stream, int* grid, DecodePlan* plan) {
  using C = Shape<D, S>;
  auto* kernel = packed_decode_kernel<T, D, S>;
  static std::atomic<int> occupancy[64];  // CTAs per SM, by device
  int occ = device >= 0 && device < 64 ? occupancy[device].load(std::memory_order_relaxed) : 0;
  if (occ == 0) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kernel, 32, C::SMEM);
    if (e != cudaSuccess) return e;
    if (occ < 1) return cudaErrorInvalidConfiguration;
    if (device >= 0 && device < 64) occupancy[device].store(occ, std::memory_order_relaxed);
  }
  p.NW = (int)std::min<int64_t>({(int64_t)occ * num_sms, kMaxPackedWorkers, p.R * p.n_layers});
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.NW);
  cfg.blockDim = dim3(32);
  cfg.dynamicSmemBytes = C::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  *grid = p.NW;
  *plan = {5, p.NW, kTile, S};
  return cudaLaunchKernelEx(&cfg, kernel, g, st, pb, p);
}

}  // namespace

cudaError_t launch_packed_decode(const Geometry& g, const Static& st, const PackedBuffers& pb, const DecodeArgs& a,
                                 int* status, int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan) {
  PackedDev p;
  p.ds = a.dstate;
  p.P = a.P;
  p.R = a.R;
  p.n_layers = a.n_layers;
  p.layer = a.layer;
  p.NW = 0;
  p.q = static_cast<const uint16_t*>(a.q);
  p.out = a.out;
  p.q_stride = a.q_layer_stride;
  p.out_stride = a.out_layer_stride;
  p.parts = a.partials;
  p.counters = a.counters;
  p.status = status;
  p.qscale = a.scale * 1.4426950408889634f;
  p.limit_ns = a.wait_limit_ns;
  p.kv_before_wait = a.kv_before_wait;
  auto by_dtype = [&](auto dc) {
    constexpr int D = decltype(dc)::value;
    return g.dtype == 1 ? launch_t<BF16T, D, kStages<D>>(g, st, pb, p, a.device, num_sms, stream, grid, plan)
                        : launch_t<F16T, D, kStages<D>>(g, st, pb, p, a.device, num_sms, stream, grid, plan);
  };
  switch (g.D) {
    case 64:
      return by_dtype(std::integral_constant<int, 64>{});
    case 80:
      return by_dtype(std::integral_constant<int, 80>{});
    case 96:
      return by_dtype(std::integral_constant<int, 96>{});
    case 128:
      return by_dtype(std::integral_constant<int, 128>{});
    default:
      return cudaErrorInvalidValue;
  }
}

}  // namespace kvc
