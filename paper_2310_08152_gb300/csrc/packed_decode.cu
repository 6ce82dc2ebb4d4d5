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
// GPU, where the beginning of a segment counts as one tile (its query, its end and its output: two thirds of one; uneven
// sequences of 64 to 4,096 rows, where the workers on short ones were the last: 187 -> 164 us).  A warp is a worker of its
// own, with a ring of stages in shared memory that 1-D bulk copies fill (codes and pairs of K and V).  A segment that spans
// several workers is joined by the last of them to finish, from parts in the workspace, in the workers' order.
//
// What bounds it: memory at 96 and 128 columns (100,003 rows of 128, two layers of 32 heads: 155 us, 6.6 TB/s); at 64 columns
// the instructions beside it (24 layers of 16 x 1,024 rows, 32 heads: 165 us, 6.1 TB/s; the copies alone 150, the arithmetic
// alone about as long).  A tile of 64 columns takes some 640 instructions of a warp, 300 of them for the codes; the pipe of
// masks and shifts is busy 54 % of the time, the tensor cores 25 %.  Tried and dropped, at 64 columns: the next tile's logits
// beside this tile's values (170 -> 175, as that leaves room for twelve workers only), 20 workers with 96 registers (185),
// codes by a conversion from 8-bit floats (its rate is that of the masks that it would save), all that a worker's first tile
// depends on in one round of loads (no change).
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>

#include "kernels.hpp"
#include "packed.cuh"
#include "tensor_core.cuh"

namespace kvc {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kTile = kPackedTile;

template <int D>
struct Shape {
  using R = PackedRow<D>;
  // Workers of an SM: the same number for each of its four schedulers, or those with more end last (10 and 13, as room for two
  // stages allowed at 128 and 96 columns, were 12 and 20 % slower).  Twelve have registers for what the compiler would like
  // (80 columns, with 16 workers and less room each: 161 us, with 12: 155 then); of 64 columns 16 were faster, 172 and 178.
  static constexpr int WARPS = D == 64 ? 16 : 12;
  // Stages of a worker: two for a tile's keys and values together, or, of 128 columns, where those leave room for 8 workers
  // only (157 us, 155 so), three for keys and values in turn.  What is read makes room for what comes S behind it.
  static constexpr bool JOINT = D != 128;
  static constexpr int S = JOINT ? 2 : 3;
  static_assert(JOINT || S % 2 == 1);
  static constexpr int KC = kTile * R::RB, KP = kTile * R::PB;
  static constexpr int HALF = KC + KP, STAGE = JOINT ? 2 * HALF : HALF;  // codes and pairs, of the keys and then of the values
  // weights times steps: [column of the operand][row of both halves of a tile] as pairs of f16, the columns 16 bytes more
  // than 128 apart, so that eight lanes' 16-byte loads meet no bank twice; the query between pieces
  static constexpr int PW = 36;
  static constexpr int PS = 4 * 8 * PW;
  static constexpr int RS = 8 * (D / 2);       // the rotation's cosines and sines at a sequence's position
  static constexpr int SMEM = S * STAGE + PS + RS + 8 * S;
  static_assert(4 * D <= PS && PS % 16 == 0);
  static_assert(WARPS * (SMEM + 1024) <= 228 * 1024);
};

struct PackedDev {
  const DState* ds;
  const int64_t* P;  // prefix sums of the sequences' places: kPackedPiece, then a tile each
  int R;             // places of a layer
  int layer;         // the first one
  int NW, share, extra;  // workers; places of each, and how many have one more, the first ones
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

// A segment among all.
struct Segment {
  int s, h, layer;
  int tiles;
  // to the next one with tiles, which exists
  __device__ __forceinline__ void advance(const int64_t* P, int H, int b) {
    if (++h < H) return;
    h = 0;
    do {
      if (++s == b) {
        s = 0;
        ++layer;
      }
      tiles = (int)(P[s + 1] - P[s]) - kPackedPiece;
    } while (tiles <= 0);
  }
};

// The worker that has the tile at place x.
__device__ __forceinline__ int worker_of(int x, const PackedDev& p) {
  const int most = p.extra * (p.share + 1);
  return x < most ? x / (p.share + 1) : p.extra + (x - most) / p.share;
}

// The sequence that holds place o of a layer: the last s with H P[s] <= o, a search of the whole warp.
__device__ __forceinline__ int seq_of(const int64_t* P, int b, int H, int o, int lane) {
  int a = 0, z = b;
  while (z - a > 1) {
    const int step = (z - a + 31) / 32, k = a + lane * step;
    const unsigned bal = __ballot_sync(kFull, k < z && H * (int)P[k] <= o);
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

__device__ __forceinline__ float warp_max(float x) {  // of the numbers among them
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
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

// 16 rows of the values' product for four columns: two of the rows in x01 (a tile's halves side by side) and x23, and the two
// eight bits up.
__device__ __forceinline__ void value_pair(float (&c)[4], uint32_t x01, uint32_t x23, uint32_t b0, uint32_t b1) {
  mma(c, low_codes(x01), high_codes(x01), low_codes(x23), high_codes(x23), b0, b1);
}

// The size of a (lo, step) pair: weights times steps have to be in f16's range, and, where lo may be far larger than the step,
// weights times lo in f32's.  And the greatest power of two that a group's sizes are taken times, 2^kMostUnit: with weights of
// 2^14 at most, products by any lo then stay finite.  (A group whose weights times sizes are all below some 2^-72, in bf16
// 2^-122, where the largest weight is 1, has fewer bits than others.)
__device__ __forceinline__ float pair_size(float2 pair, F16T) { return pair.y; }
__device__ __forceinline__ float pair_size(float2 pair, BF16T) { return fmaxf(pair.y, fabsf(pair.x) * 9.5367431640625e-7f); }  // 2^-20
template <typename T>
constexpr float kMostUnit = std::is_same_v<T, F16T> ? 60.f : 110.f;

// What a query's columns are added up times: 32 of bf16's largest are past f32's.
template <typename T>
constexpr float kQueryShare = std::is_same_v<T, F16T> ? 1.f : 0.015625f;

// The exponent of a number that is not negative; -127 of one below 2^-126.
__device__ __forceinline__ float exponent_of(float x) { return (float)((int)(__float_as_uint(x) >> 23) - 127); }
__device__ __forceinline__ float power_of_two(float e) { return __uint_as_float((uint32_t)(127 + (int)e) << 23); }  // -126 <= e

// The output row of a segment from the parts of workers first to last, in their order: each the mean of its rows' values, by
// their weights, and the sum of those.  The means come times 2^-12 of the largest sum at most, so that what is added up stays in
// range wherever the output is.  Eight parts' columns are on their way together (28 parts one by one: 2 us of 162).
template <int D>
__device__ __forceinline__ void join(const float* parts, int first, int last, float* out, int lane) {
  constexpr int QL = (D + 31) / 32;
  static_assert(kMaxPackedWorkers <= 1 << 12);
  auto from = [&](int w) { return parts + ((int64_t)w * 2 + (w == first ? 1 : 0)) * (D + 4); };
  float big = -INFINITY;
  for (int w = first + lane; w <= last; w += 32) {
    const float2 ml = __ldcg(reinterpret_cast<const float2*>(from(w)));
    big = fmaxf(big, ml.x + exponent_of(ml.y));
  }
  big = warp_max(big) + 13.f;
  float sum = 0.f, y[QL];
#pragma unroll
  for (int j = 0; j < QL; ++j) y[j] = 0.f;
  for (int w0 = first; w0 <= last; w0 += 8) {
    float f = 0.f, c[8][QL];
    const float2 ml = __ldcg(reinterpret_cast<const float2*>(from(min(w0 + (lane & 7), last))));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* a = from(min(w0 + i, last)) + 4;
#pragma unroll
      for (int j = 0; j < QL; ++j) c[i][j] = lane + 32 * j < D ? __ldcg(a + lane + 32 * j) : 0.f;
    }
    if (ml.x != -INFINITY) f = ex2(ml.x - big) * ml.y;
    if (ml.y != ml.y) f = ml.y;  // a logit that is NaN
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float fi = __shfl_sync(kFull, f, i);
      if (w0 + i > last || fi == 0.f) continue;  // a part without a weight has no mean
      sum += fi;
#pragma unroll
      for (int j = 0; j < QL; ++j) y[j] = fmaf(fi, c[i][j], y[j]);
    }
  }
  const float inv = 1.f / sum;
#pragma unroll
  for (int j = 0; j < QL; ++j)
    if (lane + 32 * j < D) out[lane + 32 * j] = y[j] * inv;
}

template <typename T, int D>
__global__ void __launch_bounds__(32, Shape<D>::WARPS)
    packed_decode_kernel(Geometry g, Static st, PackedBuffers pb, PackedDev p) {
  using C = Shape<D>;
  using R = PackedRow<D>;
  constexpr int G = R::G;
  constexpr int KW = D == 128 ? 4 : 2;              // code words of a row a lane has of the keys
  constexpr int NT = D / 16;                        // tiles of 16 columns of the values
  constexpr int QF = 2 * (D / 16);                  // registers of the query
  // Columns of the keys' other operand, of which lane t gets 2 t and 2 t + 1: with two groups, part t % 2 of each (twice, so
  // that a lane and its neighbour have all of a row's sums); with more, both parts of group t.
  constexpr bool kTwice = G == 2;
  extern __shared__ __align__(128) unsigned char smem[];
  // What comes next may be a decode that reads rows and state ahead of its own wait, which covers this kernel but not the ones
  // before it: it may start once those are complete, as they are behind a decode (kv_before_wait), or have been waited for.
  if (p.kv_before_wait) pdl_launch_dependents();
  const int lane = threadIdx.x, gr = lane >> 2, t = lane & 3, tg = t < G ? t : G - 1;
  const int wid = blockIdx.x, H = g.H;
  const int lo = wid * p.share + min(wid, p.extra), hi = lo + p.share + (wid < p.extra ? 1 : 0);

  unsigned char* ps = smem + C::S * C::STAGE;
  uint32_t* pw = reinterpret_cast<uint32_t*>(ps);
  float2* rope = reinterpret_cast<float2*>(ps + C::PS);
  uint64_t* full = reinterpret_cast<uint64_t*>(ps + C::PS + C::RS);
  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < C::S; ++i) mbar_init(&full[i], 1);
    fence_mbar_init();
  }
  fence_proxy_async_smem();
  __syncwarp();
  if (!p.kv_before_wait) {
    pdl_wait();
    pdl_launch_dependents();
  }

  Segment cs;  // of the consumed tiles
  int r;       // the next one in it
  int x = lo;  // and its place among all
  {
    cs.layer = lo / p.R;
    int o = lo - cs.layer * p.R;
    cs.s = seq_of(p.P, g.b, H, o, lane);
    const int P0 = (int)p.P[cs.s], n = (int)p.P[cs.s + 1] - P0;
    o -= H * P0;
    cs.tiles = n - kPackedPiece;
    cs.h = o / n;
    r = o - cs.h * n - kPackedPiece;
    if (r < 0) {
      x -= r;
      r = 0;
    }
  }
  if (x >= hi) return;  // a share of one that is a segment's beginning
  // The first lanes issue copies: together K codes, K pairs, V codes and V pairs one each (all by one lane: 175 us instead of
  // 171, 64 columns), in turn the first lane codes and pairs (by two: 156 instead of 155, 128 columns).  What they issue them
  // from: the segment, the next tile's place, the segment's rows from that tile on, and the first of them in the planes.
  constexpr int kFeeders = C::JOINT ? 4 : 1;
  struct {
    Segment seg;
    int rows, x;
    int64_t row;
    const unsigned char* from;  // of the lane's plane
  } feed{cs, 0, x, 0, nullptr};
  const uint32_t row_bytes = lane & 1 ? R::PB : R::RB;
  auto enter = [&](int first) {
    const DState d = p.ds[feed.seg.s];
    const int r0 = d.begin / kPackedRows * kPackedRows + first * kTile;
    feed.row = (int64_t)(p.layer + feed.seg.layer) * H * g.C + st.seq_row0[feed.seg.s] +
               (int64_t)feed.seg.h * st.cap[feed.seg.s] + r0;
    feed.rows = d.len - r0;
    if (C::JOINT) {
      const void *codes = lane & 2 ? pb.vc : pb.kc, *pairs = lane & 2 ? pb.vp : pb.kp;
      feed.from = static_cast<const unsigned char*>(lane & 1 ? pairs : codes) + feed.row * row_bytes;
    }
  };
  // the tile's keys, its values or both, after which the next tile comes
  auto issue = [&](int stage, bool keys) {
    const uint32_t n = (uint32_t)min(kTile, (feed.rows + kPackedRows - 1) & -kPackedRows);
    unsigned char* to = smem + stage * C::STAGE;
    if (lane == 0) mbar_arrive_expect_tx(&full[stage], n * (R::RB + R::PB) * (C::JOINT ? 2 : 1));
    if (C::JOINT) {
      bulk_g2s(to + (lane & 1 ? C::KC : 0) + (lane & 2 ? C::HALF : 0), feed.from, n * row_bytes, &full[stage]);
      feed.from += kTile * row_bytes;
    } else {
      bulk_g2s(to, (keys ? pb.kc : pb.vc) + feed.row * R::RB, n * R::RB, &full[stage]);
      bulk_g2s(to + C::KC, (keys ? pb.kp : pb.vp) + feed.row * R::G, n * R::PB, &full[stage]);
      if (keys) return;
      feed.row += kTile;
    }
    feed.rows -= kTile;
    ++feed.x;
    if (feed.rows > 0) return;
    feed.x += kPackedPiece;
    if (feed.x < hi) {
      feed.seg.advance(p.P, H, g.b);
      enter(0);
    }
  };
  // a decode before this one writes neither rows nor state, and did not let this one start before what wrote them was complete:
  // they may come before it is complete, while the query, the outputs and the parts may be shared with it
  if (lane < kFeeders) {
    enter(r);
    for (int i = 0; i < C::S && feed.x < hi; ++i) issue(i, C::JOINT || i % 2 == 0);
  }
  if (p.kv_before_wait) pdl_wait();

  // the query of a segment, fetched a piece ahead: columns lane + 32 j, and those they are rotated with
  constexpr int QL = (D + 31) / 32;
  float qa[QL], qb[QL];
  auto fetch_q = [&](const Segment& c) {
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
  fetch_q(cs);
  DState ds = p.ds[cs.s];
  int turned = -1;  // the sequence whose rotation is in shared memory
  int stage = 0;
  uint32_t phase = 0;
  auto next = [&]() {
    if (++stage == C::S) {
      stage = 0;
      phase ^= 1;
    }
  };
  auto arrived = [&]() { return __all_sync(kFull, mbar_wait_bounded(&full[stage], phase, p.limit_ns)); };
  // After a wait that ran out: copies that are still in flight end before their memory does.
  auto give_up = [&]() {
    if (lane == 0) {
      atomicOr(p.status, STATUS_TIMEOUT);
      for (int i = 0; i < C::S; ++i, next()) mbar_wait_bounded(&full[stage], phase, p.limit_ns);
    }
    __syncwarp();
  };

  while (x < hi) {
    // ---- a piece: tiles [r, r1) of a segment
    const int r1 = min(cs.tiles, r + hi - x);
    const int seg0 = x - r, seg1 = seg0 + cs.tiles;  // the places of the segment's tiles
    uint32_t qf[QF];  // the query as the keys' other operand
    float qsum[2];    // its sum over group t's columns, or over the first's and the second's, times qscale
    float kscale;     // of a product of codes and the query's parts
    {
      const int half = g.rot / 2;
      if (half > 0 && turned != cs.s) {  // of the sequence's heads, which come one after the other
        turned = cs.s;
        for (int k = lane; k < half; k += 32) {
          float sn, c;
          rope_sincos_full(ds.qpos, st.rope_g[k], &sn, &c);
          rope[k] = make_float2(c, sn);
        }
        __syncwarp();
      }
      float sum[QL], big = 0.f;
#pragma unroll
      for (int j = 0; j < QL; ++j) {
        const int k = lane + 32 * j;
        if (k < g.rot) {
          const float2 cs2 = rope[k < half ? k : k - half];
          qa[j] = k < half ? qa[j] * cs2.x - qb[j] * cs2.y : qa[j] * cs2.x + qb[j] * cs2.y;
        }
        sum[j] = qa[j] * kQueryShare<T>;
        big = fmaxf(big, fabsf(qa[j]));
      }
      big = warp_max(big);
#pragma unroll
      for (int i = 16; i > 0; i >>= 1) {
#pragma unroll
        for (int j = 0; j < QL; ++j) sum[j] += __shfl_xor_sync(kFull, sum[j], i);
      }
      // the largest column goes to [2^13, 2^14): it and a second part are then far from f16's ends
      // (less where the scale is so small that the products' would lose bits below 2^-126)
      const int most = min(115, (int)(__float_as_uint(p.qscale) >> 23 & 255) - 2);
      const int e = big > 0.f && big < INFINITY ? max(-115, min(most, 13 - (int)(__float_as_uint(big) >> 23) + 127)) : 0;
      const float up = __uint_as_float((uint32_t)(127 + e) << 23);
      kscale = p.qscale * __uint_as_float((uint32_t)(127 - e) << 23);
      const float sum_scale = p.qscale * (1.f / kQueryShare<T>);
      qsum[0] = qsum[1] = 0.f;
#pragma unroll
      for (int j = 0; j < QL; ++j) {
        if (kTwice)
          qsum[j & 1] = sum[j] * sum_scale;
        else if (t == j)
          qsum[0] = sum[j] * sum_scale;
      }
      __syncwarp();  // the weights of the piece before are read
#pragma unroll
      for (int j = 0; j < QL; ++j) {  // both parts of a column side by side
        const float y = qa[j] * up, h = __half2float(__float2half_rn(y));
        if (lane + 32 * j < D) pw[lane + 32 * j] = pack_halves(h, y - h);
      }
      __syncwarp();
      const int col_group = kTwice ? gr & 1 : gr >> 1;
      const uint32_t which = (kTwice ? gr & 2 : gr & 1) ? 0x7632u : 0x5410u;  // the part
      auto word = [&](int k, uint32_t* f) {
        const uint4 a = *reinterpret_cast<const uint4*>(pw + k), b = *reinterpret_cast<const uint4*>(pw + k + 4);
        const uint32_t mask = (k >> 5) == col_group ? 0xFFFFFFFFu : 0u;
        f[0] = __byte_perm(a.x, b.x, which) & mask;
        f[1] = __byte_perm(a.y, b.y, which) & mask;
        f[2] = __byte_perm(a.z, b.z, which) & mask;
        f[3] = __byte_perm(a.w, b.w, which) & mask;
      };
#pragma unroll
      for (int i = 0; i < KW; ++i) word(8 * (KW * t + i), qf + 4 * i);
      if constexpr (D == 96) word(64 + 8 * t, qf + 8);
      if constexpr (D == 80) {
        const uint4 a = *reinterpret_cast<const uint4*>(pw + 64 + 4 * t);
        const uint32_t mask = col_group == 2 ? 0xFFFFFFFFu : 0u;
        qf[8] = __byte_perm(a.x, a.z, which) & mask;
        qf[9] = __byte_perm(a.y, a.w, which) & mask;
      }
      __syncwarp();
    }
    float o[2 * NT], l = 0.f, los[G], m = -INFINITY, unit[G];
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) o[i] = 0.f;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      los[i] = 0.f;
      unit[i] = power_of_two(kMostUnit<T>);
    }

    int r0 = ds.begin / kPackedRows * kPackedRows + r * kTile;
    x += r1 - r;
    for (; r < r1; ++r, r0 += kTile) {
      // ---- a tile
      if (!arrived()) {
        give_up();
        return;  // the segment is not joined
      }
      const int k_stage = stage;
      const unsigned char* kc = smem + k_stage * C::STAGE;
      const uint32_t* kp = reinterpret_cast<const uint32_t*>(kc + C::KC);
      next();

      float z[2];  // logits of rows gr + 8 t of the tile's halves
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float v[4];  // lane t's group's part of the logits of rows gr + 8 i
        float cc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          const int row = 32 * b + 16 * a + gr;
          const unsigned char *u0 = kc + row * R::RB, *w0 = u0 + 8 * R::RB;
          float(&c)[4] = cc[a];
          if constexpr (D == 128) {
            const uint4 u = *reinterpret_cast<const uint4*>(u0 + 16 * t), w = *reinterpret_cast<const uint4*>(w0 + 16 * t);
            key_word(c, u.x, w.x, reinterpret_cast<const uint32_t(&)[4]>(qf[0]));
            key_word(c, u.y, w.y, reinterpret_cast<const uint32_t(&)[4]>(qf[4]));
            key_word(c, u.z, w.z, reinterpret_cast<const uint32_t(&)[4]>(qf[8]));
            key_word(c, u.w, w.w, reinterpret_cast<const uint32_t(&)[4]>(qf[12]));
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(u0 + 8 * t), w = *reinterpret_cast<const uint2*>(w0 + 8 * t);
            key_word(c, u.x, w.x, reinterpret_cast<const uint32_t(&)[4]>(qf[0]));
            key_word(c, u.y, w.y, reinterpret_cast<const uint32_t(&)[4]>(qf[4]));
          }
          if constexpr (D == 96)
            key_word(c, *reinterpret_cast<const uint32_t*>(u0 + 32 + 4 * t), *reinterpret_cast<const uint32_t*>(w0 + 32 + 4 * t),
                     reinterpret_cast<const uint32_t(&)[4]>(qf[8]));
          if constexpr (D == 80) {  // four columns: the second byte's go to the upper half
            const uint32_t u = __byte_perm(*reinterpret_cast<const uint16_t*>(u0 + 32 + 2 * t), 0, 0x4140);
            const uint32_t w = __byte_perm(*reinterpret_cast<const uint16_t*>(w0 + 32 + 2 * t), 0, 0x4140);
            mma(c, low_codes(u), low_codes(w), high_codes(u), high_codes(w), qf[8], qf[9]);
          }
          if (kTwice) continue;
          // a lane past the groups has a product and a sum of 0
          const float2 p0 = pair_values(kp[row * G + tg], T{}), p1 = pair_values(kp[(row + 8) * G + tg], T{});
          v[2 * a] = fmaf(p0.y, fmaf(c[0] + c[1], kscale, 8.f * qsum[0]), p0.x * qsum[0]);
          v[2 * a + 1] = fmaf(p1.y, fmaf(c[2] + c[3], kscale, 8.f * qsum[0]), p1.x * qsum[0]);
        }
        const bool odd = t & 1, two = t & 2;
        if constexpr (kTwice) {
          // lane t's row is gr + 8 t: one part of its two products is here, the other at the neighbour, whose row's part goes
          // there
          float d[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = two ? cc[1][i] : cc[0][i];
          const float s0 = (odd ? d[2] : d[0]) + __shfl_xor_sync(kFull, odd ? d[0] : d[2], 1);
          const float s1 = (odd ? d[3] : d[1]) + __shfl_xor_sync(kFull, odd ? d[1] : d[3], 1);
          const uint2 kpair = *reinterpret_cast<const uint2*>(kp + 2 * (32 * b + 8 * t + gr));
          const float2 p0 = pair_values(kpair.x, T{}), p1 = pair_values(kpair.y, T{});
          z[b] = fmaf(p0.y, fmaf(s0, kscale, 8.f * qsum[0]), p0.x * qsum[0]) +
                 fmaf(p1.y, fmaf(s1, kscale, 8.f * qsum[1]), p1.x * qsum[1]);
        } else {
          // the sum over the groups; lane t is left with row gr + 8 t
          const float s0 = (odd ? v[1] : v[0]) + __shfl_xor_sync(kFull, odd ? v[0] : v[1], 1);
          const float s1 = (odd ? v[3] : v[2]) + __shfl_xor_sync(kFull, odd ? v[2] : v[3], 1);
          z[b] = (two ? s1 : s0) + __shfl_xor_sync(kFull, two ? s0 : s1, 2);
        }
      }

      if (!C::JOINT && !arrived()) {
        give_up();
        return;
      }
      const int v_stage = C::JOINT ? k_stage : stage;
      const unsigned char* vc = smem + v_stage * C::STAGE + (C::JOINT ? C::HALF : 0);
      const uint32_t* vp = reinterpret_cast<const uint32_t*>(vc + C::KC);
      if (!C::JOINT) next();
      uint32_t vpair[2][G];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < G; ++i) vpair[b][i] = vp[(32 * b + 8 * t + gr) * G + i];
      if (r0 < ds.begin || r0 + kTile > ds.len || (ds.mask_lo < r0 + kTile && ds.mask_hi > r0)) {  // not all of it is seen
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int at = r0 + 32 * b + 8 * t + gr;
          if (at >= ds.begin && at < ds.len && !(at >= ds.mask_lo && at < ds.mask_hi)) continue;
          z[b] = -INFINITY;
#pragma unroll
          for (int i = 0; i < G; ++i) vpair[b][i] = 0;
        }
      }
      // A row's weight is 2^(10 - m) times what it would be without a reference, m a whole number that the logits do not pass by
      // more than 4.  Each group's sums go by a power of two of their own besides, unit[i], so that the largest product of a
      // weight and a pair's size among the rows so far is some 2^10 whatever the groups' sizes are and however they change along
      // the rows: unit[i] falls where a row's product would pass 2^14, and rises as m does, which makes the weights of the rows
      // before smaller.  (Taken from a piece's first rows alone, it left weights of 2^-40 beside pairs that became 2^40 times
      // as large: no bits of the other groups.)  A group without a size yet has the greatest one.  Pairs that are NaN do not
      // count.
      float e[2], w[2][G], x01[2][G];  // weights; times the groups' powers of two; times steps
      auto weigh = [&]() -> float {  // the largest of what has to stay in range
        const float ref = m == -INFINITY ? 10.f : 10.f - m;
        float most = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          e[b] = ex2(z[b] + ref);
          most = fmaxf(most, e[b]);
#pragma unroll
          for (int i = 0; i < G; ++i) {
            const float2 pv = pair_values(vpair[b][i], T{});
            w[b][i] = e[b] * unit[i];
            x01[b][i] = w[b][i] * pv.y;
            most = fmaxf(most, w[b][i] * pair_size(pv, T{}));
          }
        }
        return most;
      };
      const bool begins = m == -INFINITY;  // nothing but 0 or NaN is summed yet
      const float most = warp_max(weigh());
      if (begins || most > 16384.f) {
        const float m_new = fmaxf(m, ceilf(warp_max(fmaxf(z[0], z[1])))), up = begins ? INFINITY : m_new - m;
        float f = 1.f;  // group t's
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const float s0 = pair_size(pair_values(vpair[0][i], T{}), T{}), s1 = pair_size(pair_values(vpair[1][i], T{}), T{});
          const float top = ceilf(warp_max(fmaxf(z[0] + exponent_of(s0), z[1] + exponent_of(s1))));
          const float was = exponent_of(unit[i]), now = fmaxf(fminf(fminf(was + up, kMostUnit<T>), m_new - top), -126.f);
          const float fi = ex2(now - was - up);
          unit[i] = power_of_two(now);
          los[i] *= fi;
          if (t == i) f = fi;
        }
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) o[i] *= f;
        l *= ex2(-up);
        m = m_new;
        weigh();
      }
      l += e[0] + e[1];
      const int at = 8 * (gr & 3) + 2 * t + (gr >> 2);  // of row i = gr + 8 t of the halves: 8 (i % 4) + i / 4
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const float x0 = x01[0][i], x1 = x01[1][i];
        los[i] = fmaf(8.f, x0 + x1, fmaf(w[0][i], pair_values(vpair[0][i], T{}).x, fmaf(w[1][i], pair_values(vpair[1][i], T{}).x, los[i])));
        const uint32_t h = pack_halves(x0, x1);
        const float2 back = F16T::f2(h);
        pw[2 * i * C::PW + at] = h;
        pw[(2 * i + 1) * C::PW + at] = pack_halves(x0 - back.x, x1 - back.y);
      }
      __syncwarp();
      if (!C::JOINT && lane < kFeeders && feed.x < hi) issue(k_stage, false);  // the keys are read: S is odd

      float acc[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // rows t + 8 k and t + 8 k + 4 of both halves
        const uint2 w = *reinterpret_cast<const uint2*>(pw + gr * C::PW + 8 * t + 2 * k);
        const unsigned char* u = vc + (8 * k + t) * R::RB;
        auto word = [&](int i, uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3) {
          uint32_t y = __byte_perm(w0, w1, 0x5410), v = __byte_perm(w2, w3, 0x5410);
          value_pair(acc[i], y, v, w.x, w.y);
          value_pair(acc[i + 1], y >> 8, v >> 8, w.x, w.y);
          y = __byte_perm(w0, w1, 0x7632), v = __byte_perm(w2, w3, 0x7632);
          value_pair(acc[i + 2], y, v, w.x, w.y);
          value_pair(acc[i + 3], y >> 8, v >> 8, w.x, w.y);
        };
        constexpr int HALF = 32 * R::RB, NEXT = 4 * R::RB;
        if constexpr (D == 128) {
          auto at2 = [&](int j) { return *reinterpret_cast<const uint2*>(u + j + 8 * gr); };
          const uint2 w0 = at2(0), w1 = at2(HALF), w2 = at2(NEXT), w3 = at2(HALF + NEXT);
          word(0, w0.x, w1.x, w2.x, w3.x);
          word(4, w0.y, w1.y, w2.y, w3.y);
        } else {
          auto at1 = [&](int j) { return *reinterpret_cast<const uint32_t*>(u + j + 4 * gr); };
          word(0, at1(0), at1(HALF), at1(NEXT), at1(HALF + NEXT));
        }
        if constexpr (D == 96) {  // the last four words, half a word a lane
          auto at1 = [&](int j) { return (uint32_t)*reinterpret_cast<const uint16_t*>(u + j + 32 + 2 * gr); };
          const uint32_t y = __byte_perm(at1(0), at1(HALF), 0x5410), v = __byte_perm(at1(NEXT), at1(HALF + NEXT), 0x5410);
          value_pair(acc[4], y, v, w.x, w.y);
          value_pair(acc[5], y >> 8, v >> 8, w.x, w.y);
        }
        if constexpr (D == 80) {  // the last two, a byte a lane
          auto at1 = [&](int j) { return (uint32_t)u[j + 32 + gr]; };
          value_pair(acc[4], at1(0) | at1(HALF) << 16, at1(NEXT) | at1(HALF + NEXT) << 16, w.x, w.y);
        }
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        o[2 * i] += acc[i][0] + acc[i][1];
        o[2 * i + 1] += acc[i][2] + acc[i][3];
      }
      __syncwarp();  // the values and the weights are read
      if (lane < kFeeders && feed.x < hi) issue(v_stage, true);
    }

    // ---- the end of a piece
    const Segment was = cs;
    x += kPackedPiece;
    if (x < hi) {
      cs.advance(p.P, H, g.b);
      fetch_q(cs);
      if (cs.s != was.s) ds = p.ds[cs.s];
    }
    r = 0;
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
    float mine = los[0], scale = unit[0];  // group t's
#pragma unroll
    for (int k = 1; k < G; ++k)
      if (t == k) {
        mine = los[k];
        scale = unit[k];
      }
    scale = __uint_as_float((254u << 23) - __float_as_uint(scale));  // 1 / scale, a power of two
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < 2 * NT; ++i) o[i] = (o[i] + mine) * inv * scale;
    float* orow = p.out + (int64_t)was.layer * p.out_stride + ((int64_t)was.s * H + was.h) * D;
    if (seg0 >= lo && seg1 <= hi) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
        if (t == col(i) / 32) {
          orow[col(i)] = o[2 * i];
          orow[col(i) + 1] = o[2 * i + 1];
        }
      continue;
    }
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
    const int first = worker_of(seg0, p), last = worker_of(seg1 - 1, p);
    __syncwarp();
    int done = 0;
    if (lane == 0) {  // the warp's part is visible before the count, the others' after it
      __threadfence();
      done = atomicAdd(p.counters + first, 1) == last - first;
      if (done) __threadfence();
    }
    if (!__shfl_sync(kFull, done, 0)) continue;
    __syncwarp();
    join<D>(p.parts, first, last, orow, lane);
    if (lane == 0) p.counters[first] = 0;
  }
}

template <typename T, int D>
cudaError_t launch_t(const Geometry& g, const Static& st, const PackedBuffers& pb, PackedDev p, int64_t places, int device,
                     int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan) {
  using C = Shape<D>;
  auto* kernel = packed_decode_kernel<T, D>;
  static std::atomic<int> occupancy[64];  // workers of an SM, by device
  int occ = device >= 0 && device < 64 ? occupancy[device].load(std::memory_order_relaxed) : 0;
  if (occ == 0) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kernel, 32, C::SMEM);
    if (e != cudaSuccess) return e;
    if (occ < 1) return cudaErrorInvalidConfiguration;
    occ = std::min(occ, C::WARPS);
    if (device >= 0 && device < 64) occupancy[device].store(occ, std::memory_order_relaxed);
  }
  p.NW = (int)std::min<int64_t>({(int64_t)occ * num_sms, kMaxPackedWorkers, places});
  p.share = (int)(places / p.NW);
  p.extra = (int)(places % p.NW);
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
  *plan = {5, p.NW, kTile, C::S};
  return cudaLaunchKernelEx(&cfg, kernel, g, st, pb, p);
}

}  // namespace

cudaError_t launch_packed_decode(const Geometry& g, const Static& st, const PackedBuffers& pb, const DecodeArgs& a,
                                 int* status, int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan) {
  PackedDev p;
  p.ds = a.dstate;
  p.P = a.P;
  const int64_t places = a.R * a.n_layers;
  if (places > INT32_MAX) return cudaErrorInvalidValue;  // 10 TB of rows
  p.R = (int)a.R;
  p.layer = a.layer;
  p.NW = p.share = p.extra = 0;
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
    return g.dtype == 1 ? launch_t<BF16T, D>(g, st, pb, p, places, a.device, num_sms, stream, grid, plan)
                        : launch_t<F16T, D>(g, st, pb, p, places, a.device, num_sms, stream, grid, plan);
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
