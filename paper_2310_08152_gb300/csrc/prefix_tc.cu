// The prefix part of a shared-prefix decode for large groups, on the fifth-generation tensor cores: up to 128 members'
// queries of one (layer, head) against a run of the prefix's rows.  What it computes and leaves is prefix_kernel's
// (prefix.cu); past 32 members the 16 x 8 x 16 instructions bound that kernel (64 samples of 32,768 rows, two layers of 32
// heads of 128, bf16: 312 us, its tensor pipe at 54 %, where the rows' bytes take 158; here 206), and these do four times as much.
//
// One CTA per SM.  Per tile of 128 rows: S = Q K^T into one of two TMEM buffers; eight warps take it, a query per thread
// pair and 64 columns each, agree on the row's maximum through shared memory, and leave P in TMEM, as two 16-bit parts in
// f16 (22 bits) and three in bf16 (24): the first two over S, the third beside it.  The product of the next tile goes ahead
// of P V of this one.  P's reference is kept as in prefix_kernel, so that O is rarely scaled.  K and V come by TMA through
// rings of two tiles; the queries, whose rows are anywhere in the batch, are gathered (and rotated) by the warps.  Rows of
// V past the run's end are zeroed in shared memory, for whatever they hold would meet P = 0.
//
// The tensor core cuts what it adds rather than round it (16,384 rows in one sum: an error of 1.2e-5 of the output's
// norm), so each tile's P V is a sum of its own, the small parts first, which the warps add to their columns of O in
// registers: errors of 4e-7 to 9e-7, where two parts and sums of 2,048 rows in TMEM left 1.3e-6 to 4.6e-6 in bf16.  The
// call of the case above, with two own rows a sample, takes 218 us (206 with two parts and long sums), in f16 192 (207); 4
// layers of 32 heads of 64 in bf16 385 (325).  P written 32 columns at a time instead of 16 spills registers: 243.
// What bounds it: the products (the tensor pipe is at 56 % in that case) and the warps that make P, a third part of it in
// bf16, by turns; HBM is at 5.2 TB/s.
#include <cuda.h>

#include <atomic>
#include <cstring>

#include "device_common.cuh"
#include "kernels.hpp"
#include "tensor_core.cuh"

namespace kvc {
namespace {

constexpr int kRows = 128;  // queries of a CTA, rows of a tile
constexpr int kPWarps = 8;
constexpr int kPThreads = kPWarps * 32;
constexpr int kTcThreads = kPThreads + 64;
template <int D, int NQ, int NP>
struct TcCfg {
  static constexpr int SW = (2 * D) % 128 == 0 ? 128 : (2 * D) % 64 == 0 ? 64 : 32;
  static constexpr int SUB = SW / 2;
  static constexpr int NSUB = D / SUB;
  static constexpr uint32_t SUBB = kRows * SW;
  static constexpr uint32_t TILE = kRows * D * 2;
  // stages of K and of V: with three parts of the queries at 128 columns there is room for one of V
  static constexpr int KST = 2;
  static constexpr int VST = TILE * (NQ + 4) + 1024 > 222 * 1024 ? 1 : 2;
  static constexpr uint32_t K_OFF = TILE * NQ;
  static constexpr uint32_t V_OFF = K_OFF + KST * TILE;
  static constexpr uint32_t SMEM = V_OFF + VST * TILE + 1024;  // + aligning the base
  // TMEM columns: two S tiles, each taken over by the first two parts of its P, the third parts, then O of a tile
  static constexpr uint32_t P2_COL = 256;
  static constexpr uint32_t O_COL = P2_COL + (NP > 2 ? 2 * 64 : 0);
  static_assert(SMEM <= 227 * 1024 - 3584 && O_COL + D <= 512, "shared memory, TMEM");
};

template <typename T, int D, int NQ>
__global__ void __launch_bounds__(kTcThreads, 1)
    prefix_tc_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const PrefixArgs p) {
  constexpr int NP = kFullParts<T>;  // of P
  using Cf = TcCfg<D, NQ, NP>;
  constexpr int SW = Cf::SW, SUB = Cf::SUB, KST = Cf::KST, VST = Cf::VST, CH = D / 8;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t k_full[KST], k_empty[KST], v_full[VST], v_empty[VST], s_full[2], q_full, p_full, pv_done;
  __shared__ uint32_t tmem_slot;
  __shared__ float s_max[2][2][kRows];
  __shared__ float s_sum[kRows];
  const uint32_t sm = (smem_addr(raw) + 1023u) & ~1023u;
  unsigned char* smp = raw + (sm - smem_addr(raw));
  const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31, tid = threadIdx.x;
  const uint32_t limit_ns = (uint32_t)p.wait_limit_ns;
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 32) {
    for (int i = 0; i < KST; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < VST; ++i) {
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    mbar_init(&s_full[0], 1);
    mbar_init(&s_full[1], 1);
    mbar_init(&q_full, kPThreads);
    mbar_init(&p_full, kPThreads);
    mbar_init(&pv_done, 1);
    fence_mbar_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();               // q and the prefix's rows come from earlier kernels
  pdl_launch_dependents();  // as in prefix_kernel; this CTA has its TMEM
  const int lh = (int)(blockIdx.x / (unsigned)p.n_units);
  const PrefixUnit un = p.units[blockIdx.x - lh * p.n_units];
  const int layer = lh / p.H, h = lh - layer * p.H;
  const int n_keys = un.key1 - un.key0, n_tiles = (n_keys + kRows - 1) / kRows;
  bool ok = true;

  if (warp == kPWarps) {
    // ---------------- loads ----------------
    if (lane == 0) {
      const int row0 = (int)((int64_t)(p.layer + layer) * p.H * p.C + p.st.seq_row0[un.s]) + h * p.st.cap[un.s] + un.key0;
      int nk = 0, nv = 0;
      for (int t = 0; ok && t < n_tiles; ++t) {
        const int ks = t % KST, vs = t % VST;
        if (t >= KST && !(ok = pf_wait(&k_empty[ks], (t / KST & 1) ^ 1, limit_ns))) break;
        mbar_arrive_expect_tx(&k_full[ks], Cf::TILE);
#pragma unroll
        for (int i = 0; i < Cf::NSUB; ++i)
          tma_load_2d(sm + Cf::K_OFF + ks * Cf::TILE + i * Cf::SUBB, &mk, i * SUB, row0 + t * kRows, &k_full[ks]);
        ++nk;
        if (t >= VST && !(ok = pf_wait(&v_empty[vs], (t / VST & 1) ^ 1, limit_ns))) break;
        mbar_arrive_expect_tx(&v_full[vs], Cf::TILE);
#pragma unroll
        for (int i = 0; i < Cf::NSUB; ++i)
          tma_load_2d(sm + Cf::V_OFF + vs * Cf::TILE + i * Cf::SUBB, &mv, i * SUB, row0 + t * kRows, &v_full[vs]);
        ++nv;
      }
      // never leave with copies in flight
      for (int u = max(nk - KST, 0); u < nk; ++u) (void)pf_wait(&k_full[u % KST], u / KST & 1, limit_ns);
      for (int u = max(nv - VST, 0); u < nv; ++u) (void)pf_wait(&v_full[u % VST], u / VST & 1, limit_ns);
    }
    __syncwarp();
  } else if (warp == kPWarps + 1) {
    // ---------------- products ----------------
    constexpr uint32_t idS = mma_idesc(Pack16<T>::kType, 0, kRows, kRows);
    constexpr uint32_t idO = mma_idesc(Pack16<T>::kType, 1, kRows, D);
    constexpr uint32_t SBO = 8 * SW;
    auto uni_wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(0xFFFFFFFFu, pf_wait(bar, parity, limit_ns)); };
    const uint32_t q_d = desc_lo(sm, 16);
    auto issue_s = [&](int t) -> bool {
      // the buffer was P's of tile t - 2, whose product was issued before this one and goes first
      const int st = t % KST, sb = t & 1;
      if (!uni_wait(&k_full[st], t / KST & 1)) return false;
      tc_fence_after();
      const uint32_t k_d = desc_lo(sm + Cf::K_OFF + st * Cf::TILE, 16);
      if (elect_one()) {
#pragma unroll
        for (int part = NQ - 1; part >= 0; --part) {  // the small parts first: what is added to a sum is cut
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            const uint32_t off = ((kk * 16) / SUB * Cf::SUBB + (kk * 16) % SUB * 2) >> 4;
            tc_mma(tmem + sb * kRows, desc(q_d + part * (Cf::TILE >> 4) + off, SBO, SW), desc(k_d + off, SBO, SW), idS, part < NQ - 1 || kk > 0);
          }
        }
        tc_commit(&s_full[sb]);
        tc_commit(&k_empty[st]);
      }
      __syncwarp();
      return true;
    };
    ok = uni_wait(&q_full, 0);
    if (ok) ok = issue_s(0);
    for (int t = 0; ok && t < n_tiles; ++t) {
      if (t + 1 < n_tiles && !(ok = issue_s(t + 1))) break;
      const int st = t % VST;
      if (!(ok = uni_wait(&v_full[st], t / VST & 1))) break;
      if (!(ok = uni_wait(&p_full, t & 1))) break;
      fence_proxy_async_smem();  // rows of V zeroed through the generic proxy
      tc_fence_after();
      const uint32_t v_d = desc_lo(sm + Cf::V_OFF + st * Cf::TILE, Cf::SUBB);
      if (elect_one()) {
#pragma unroll
        for (int part = NP - 1; part >= 0; --part) {
          const uint32_t p_col = part < 2 ? (t & 1) * kRows + part * 64 : Cf::P2_COL + (t & 1) * 64;
#pragma unroll
          for (int kk = 0; kk < kRows / 16; ++kk)
            tc_mma_ts(tmem + Cf::O_COL, tmem + p_col + 8 * kk, desc(v_d + kk * SW, SBO, SW), idO, part < NP - 1 || kk > 0);
        }
        tc_commit(&pv_done);
        tc_commit(&v_empty[st]);
      }
      __syncwarp();
    }
  } else {
    // ---------------- the queries, then P ----------------
    const int half = warp >> 2, r = (warp & 3) * 32 + lane;  // columns [64 half, 64 half + 64) of query r
    // 16-byte chunk c of row x, in the tile's swizzle
    auto at = [&](int x, int c) -> uint32_t {
      const int cps = SW / 16, sub = c / cps, cc = c % cps;
      const int mix = SW == 128 ? x & 7 : SW == 64 ? x >> 1 & 3 : x >> 2 & 1;
      return sub * Cf::SUBB + x * SW + ((cc ^ mix) << 4);
    };
    for (int x = tid; x < kRows * CH; x += kPThreads) {
      const int row = x / CH, c = x % CH;
      uint32_t part[NQ][4];
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[i][e] = 0;
      if (row < un.n_mem) {
        const int s = p.members[un.mem0 + row];
        const uint16_t* q = p.q + (int64_t)layer * p.q_stride + ((int64_t)s * p.H + h) * D;
        query_chunk<T, NQ>(q, c, p.rot, NQ > 1 ? p.ds[s].qpos : 0, p.st.rope_g, part);
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        *reinterpret_cast<uint4*>(smp + i * Cf::TILE + at(row, c)) = make_uint4(part[i][0], part[i][1], part[i][2], part[i][3]);
    }
    fence_proxy_async_smem();
    mbar_arrive(&q_full);

    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const bool live = r < un.n_mem;
    const int member = live ? p.members[un.mem0 + r] : 0;
    float* to = p.parts + (((int64_t)layer * p.n_parts + p.split0[member] + un.split) * p.H + h) * (D + 4);
    float m = -INFINITY, l = 0.f;
    // the thread's columns of O, 16 at a time: chunks half, half + 2, ..
    constexpr int OC = (D / 16 + 1) / 2;
    float o[OC][16];
#pragma unroll
    for (int c = 0; c < OC; ++c)
#pragma unroll
      for (int x = 0; x < 16; ++x) o[c][x] = 0.f;
    auto add_o = [&]() {
#pragma unroll
      for (int c = 0; c < OC; ++c) {
        if (half + 2 * c >= D / 16) break;
        float v[16];
        tmem_ld16(tmem + lanes + Cf::O_COL + (half + 2 * c) * 16, v);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
          const float2 sum = __fadd2_rn(make_float2(o[c][x], o[c][x + 1]), make_float2(v[x], v[x + 1]));
          o[c][x] = sum.x;
          o[c][x + 1] = sum.y;
        }
      }
    };
    for (int t = 0; t < n_tiles; ++t) {
      float s[64];
      const int sb = t & 1;
      if (ok) ok = __all_sync(0xFFFFFFFFu, pf_wait(&s_full[sb], t / 2 & 1, limit_ns));
      tc_fence_after();
      if (ok) {
        tmem_ld32(tmem + lanes + sb * kRows + half * 64, s);
        tmem_ld32(tmem + lanes + sb * kRows + half * 64 + 32, s + 32);
        tmem_wait_ld();
      }
      const int left = n_keys - t * kRows - half * 64;  // the thread's columns that are rows of the run
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (ok) {
        const float2 cc = make_float2(p.c2, p.c2);
#pragma unroll
        for (int x = 0; x < 64; x += 2) {
          const float2 z = __fmul2_rn(make_float2(s[x], s[x + 1]), cc);
          s[x] = z.x;
          s[x + 1] = z.y;
        }
        if (left < 64) {
#pragma unroll
          for (int x = 0; x < 64; ++x)
            if (x >= left) s[x] = -INFINITY;
        }
#pragma unroll
        for (int x = 0; x < 64; x += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], s[x + e]);
      }
      float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      s_max[sb][half][r] = top;
      tc_fence_before();
      bar_sync(1, kPThreads);
      top = fmaxf(top, s_max[sb][half ^ 1][r]);
      float scale = 1.f;
      const bool moved = top > m + 14.f;
      if (moved) {
        const float to = top - 6.f;
        scale = m == -INFINITY ? 0.f : ex2(m - to);
        m = to;
      }
      const float mu = m == -INFINITY ? 0.f : m;
      if (ok) {
        float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
        tc_fence_after();
        // the first two parts over S, which both halves have read by now
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t pp[NP][8];
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            const int e = 16 * c + 2 * x;
            const float2 w = make_float2(ex2(s[e] - mu), ex2(s[e + 1] - mu));
            if (x & 1)
              sum1 = __fadd2_rn(sum1, w);
            else
              sum0 = __fadd2_rn(sum0, w);
            uint32_t part[NP];
            split_parts<T, NP>(w.x, w.y, part);
#pragma unroll
            for (int i = 0; i < NP; ++i) pp[i][x] = part[i];
          }
#pragma unroll
          for (int i = 0; i < NP; ++i)
            tmem_st8u(tmem + lanes + (i < 2 ? sb * kRows + i * 64 : Cf::P2_COL + sb * 64) + half * 32 + 8 * c, pp[i]);
        }
        l = l * scale + ((sum0.x + sum0.y) + (sum1.x + sum1.y));
        // O is free once that of the tile before is taken
        if (t > 0) ok = __all_sync(0xFFFFFFFFu, pf_wait(&pv_done, (t - 1) & 1, limit_ns));
      }
      if (ok) {
        tc_fence_after();
        if (t > 0) add_o();
        if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
          for (int c = 0; c < OC; ++c)
#pragma unroll
            for (int x = 0; x < 16; ++x) o[c][x] *= scale;
        }
        if (t + 1 == n_tiles && n_keys % kRows != 0) {  // rows of V past the end
          const int st = t % VST, from = n_keys % kRows;
          ok = __all_sync(0xFFFFFFFFu, pf_wait(&v_full[st], t / VST & 1, limit_ns));
          if (ok) {
            constexpr int CPS = SW / 16;
            for (int x = tid; x < (kRows - from) * CH; x += kPThreads) {
              const int row = from + x / CH, c = x % CH;
              *reinterpret_cast<uint4*>(smp + Cf::V_OFF + st * Cf::TILE + c / CPS * Cf::SUBB + row * SW + c % CPS * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
          }
        }
        tmem_wait_st();
      }
      tc_fence_before();
      mbar_arrive(&p_full);
    }
    if (ok) ok = __all_sync(0xFFFFFFFFu, pf_wait(&pv_done, (n_tiles - 1) & 1, limit_ns));
    if (half) s_sum[r] = l;
    bar_sync(1, kPThreads);
    tc_fence_after();
    if (ok) {
      add_o();
      if (live) {
        if (!half) *reinterpret_cast<float4*>(to) = make_float4(m, l + s_sum[r], 0.f, 0.f);
#pragma unroll
        for (int c = 0; c < OC; ++c) {
          if (half + 2 * c >= D / 16) break;
          float4* at = reinterpret_cast<float4*>(to + 4 + (half + 2 * c) * 16);
#pragma unroll
          for (int x = 0; x < 4; ++x) at[x] = make_float4(o[c][4 * x], o[c][4 * x + 1], o[c][4 * x + 2], o[c][4 * x + 3]);
        }
      }
    }
  }
  if (!ok) atomicOr(p.status, STATUS_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

template <typename T, int D, int NQ>
cudaError_t launch_tc_t(const PrefixMaps& maps, const PrefixArgs& a, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!done[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(prefix_tc_kernel<T, D, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TcCfg<D, NQ, kFullParts<T>>::SMEM);
    if (e != cudaSuccess) return e;
    done[dev].store(true, std::memory_order_release);
  }
  CUtensorMap mk, mv;
  std::memcpy(&mk, maps.k, sizeof mk);
  std::memcpy(&mv, maps.v, sizeof mv);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)a.n_units * a.H * a.n_layers));
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = TcCfg<D, NQ, kFullParts<T>>::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, prefix_tc_kernel<T, D, NQ>, mk, mv, a);
}

}  // namespace

cudaError_t launch_prefix_tc(const Geometry& g, const PrefixMaps& maps, const PrefixArgs& a, cudaStream_t stream) {
  if (a.n_units <= 0) return cudaSuccess;
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (g.dtype == 1) return g.rot > 0 ? launch_tc_t<BF16T, D, 3>(maps, a, stream) : launch_tc_t<BF16T, D, 1>(maps, a, stream);
    return g.rot > 0 ? launch_tc_t<F16T, D, 2>(maps, a, stream) : launch_tc_t<F16T, D, 1>(maps, a, stream);
  };
  switch (g.D) {
    case 64:
      return go(std::integral_constant<int, 64>{});
    case 80:
      return go(std::integral_constant<int, 80>{});
    case 96:
      return go(std::integral_constant<int, 96>{});
    case 128:
      return go(std::integral_constant<int, 128>{});
    default:
      return cudaErrorInvalidValue;
  }
}

}  // namespace kvc
