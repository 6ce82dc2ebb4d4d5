// Attention weights of a prompt's queries, summed for each key: what the scores of a prompt's rows are made of.
//
//   score_i += sum over the queries t that see row i of  2^(z_ti - L_t),   z_ti = scale log2(e) <q_t, k_i>,
//   L_t = log2 sum over the rows that t sees of 2^z_ti
//
// in two passes over the products of queries and keys on the tensor cores (tcgen05, accumulators in TMEM, operands by
// TMA): keeping z between them would write and read 4 bytes a pair where the product costs d_head multiply-adds.
//
//   pass 0   S = Q K^T, a query per thread and a key per column: the running maximum and sum of each query.  A unit is
//            128 queries of one head against some key tiles (all, or a part where the units are few).
//   pass 1   S^T = K Q^T, a key per thread and a query per column, so that a key's sum over the queries stays in one
//            thread's register: no shuffles, no atomics, one addition to the score at the end.  A unit is some key tiles
//            of one head against every query tile that sees them; where there is one query tile, it stays and the key
//            tiles stream by (few), else the key tile stays and the query tiles stream by.
//
// Mask: row i is visible to the query at stored row t exactly when i <= t <= hid(i), except that a <CL> query sees only
// itself.
//
// Eight warps take S from TMEM (two buffers of 128 columns), so that four warps per scheduler hide each other's latencies
// (four warps a CTA, two per scheduler: 325 us on OPT-1.3B-shaped prompts): in pass 0 64 columns each, in pass 1 four of
// them each step by turns, which leaves no barrier between all of them but one per key tile (64 columns each there too:
// 216 us, and 119 for the window of 64 queries); one loads the tiles and one
// issues the products.  A mask is a bit per column, looked at where a bit is missing.
// Rotated queries come from a kernel of their own as two (f16) or three (bf16) 16-bit parts, each a product of its own.
// What bounds it: the exponentials, two a pair, and the instructions around them, for whole prompts also of hidden pairs:
// every 64 columns with a visible pair are worked on whole (four prompts of 2,048 tokens whose spans still hold half of
// the rows, 32 heads: 2.85e8 pairs, 1.29e8 of them visible, 191 us); for windows HBM, K being read by both passes
// (six prompts of 3,000 to 8,191 rows, 64 queries, d_head 128: 94 us, the bytes of K once 41).
#include <cuda.h>

#include <atomic>
#include <cstring>

#include "device_common.cuh"
#include "kernels.hpp"
#include "tensor_core.cuh"

namespace kvc {
namespace {

constexpr int kSWarps = 8;  // warps that take S
constexpr int kSThreads = kSWarps * 32;
constexpr int kScThreads = kSThreads + 64;
constexpr int kRows = 128;  // queries, and keys, of a tile

// kLse16 is the first pass of windows of up to 16 queries, which are the columns there too; kSumFew takes them and windows
// of up to 128.
enum Pass { kLse = 0, kSumFew = 1, kSumMany = 2, kLse16 = 3 };

// NQ 16-bit parts of a query, QN queries of a tile.
template <int D, int NQ, int PASS, int QN>
struct ScCfg {
  static constexpr int SW = (2 * D) % 128 == 0 ? 128 : (2 * D) % 64 == 0 ? 64 : 32;
  static constexpr int SUB = SW / 2;
  static constexpr int NSUB = D / SUB;
  static constexpr uint32_t SUBB = kRows * SW;
  static constexpr uint32_t TILE = kRows * D * 2;
  static constexpr uint32_t QSUBB = QN * SW;
  static constexpr uint32_t QTILE = QN * D * 2;
  static constexpr uint32_t QT = QTILE * NQ;  // a query tile's parts
  // Stages: as many as two CTAs per SM leave room for, three at most, and where fewer than `least` would be left as many
  // as one CTA has room for.
  static constexpr uint32_t ROOM = 110 * 1024, ALL = 220 * 1024;
  static constexpr int fit(uint32_t fixed, uint32_t each, int least) {
    for (int n = 3; n >= least; --n)
      if (fixed + n * each <= ROOM) return n;
    for (int n = 3; n > 1; --n)
      if (fixed + n * each <= ALL) return n;
    return 1;
  }
  static constexpr int KS = PASS == kSumMany ? 1 : fit(QT, TILE, 2);
  static constexpr int QS = PASS == kSumMany ? fit(TILE, QT, 1) : 1;
  static constexpr uint32_t Q_OFF = KS * TILE;
  static constexpr uint32_t NEED = Q_OFF + QS * QT + 1024;  // + aligning the base
  // no third CTA on an SM, which would wait for columns of TMEM
  static constexpr uint32_t SMEM = NEED < 80 * 1024 ? 80 * 1024 : NEED;
  static constexpr int CPS = SMEM <= ROOM + 1024 ? 2 : 1;
  static_assert(SMEM <= 227 * 1024, "shared memory");
};

template <typename T, int D, int NQ, int PASS, int QN>
__global__ void __launch_bounds__(kScThreads, ScCfg<D, NQ, PASS, QN>::CPS)
    score_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mq,
                 const __grid_constant__ CUtensorMap mq1, const __grid_constant__ CUtensorMap mq2, const ScoreArgs a) {
  using Cf = ScCfg<D, NQ, PASS, QN>;
  constexpr int KS = Cf::KS, QS = Cf::QS;
  extern __shared__ unsigned char raw[];
  __shared__ __align__(8) uint64_t k_full[KS], k_empty[KS], q_full[QS], q_empty[QS], s_full[2], s_empty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(16) float s_neg[2][kRows];  // pass 1: -L of a tile's queries
  __shared__ __align__(16) uint32_t s_none[2][4];  // which of them have no part in the sums: <CL>, none and s_bad
  __shared__ __align__(16) uint32_t s_bad[2][4];   // whose weights are not numbers
  __shared__ __align__(16) uint32_t s_cl[2][4];    // <CL>
  __shared__ float2 s_half[kRows];                 // results of the upper columns (kLse16: of 16 queries by eight warps)
  const uint32_t sm = (smem_addr(raw) + 1023u) & ~1023u;
  const int warp = uniform((int)(threadIdx.x >> 5)), lane = threadIdx.x & 31, tid = threadIdx.x;
  const uint32_t limit_ns = (uint32_t)a.wait_limit_ns;
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(256u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 32) {
    for (int i = 0; i < KS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
    }
    for (int i = 0; i < QS; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_empty[i], PASS == kLse ? kSThreads : kSThreads / 2);
    }
    fence_mbar_init();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Not before this CTA has its columns of TMEM: a CTA of the second pass that took them would wait for this one.
  pdl_launch_dependents();
  const uint32_t tmem = tmem_slot;
  const int item = (int)(blockIdx.x / (unsigned)a.H), h = (int)(blockIdx.x - (unsigned)item * a.H);
  const ScoreUnit un = a.units[item];
  const ScoreSeq& sq = un.q;
  const int nqt = (sq.len - sq.q0 + kRows - 1) / kRows;
  // the query tiles of key tile kt: those that end at or after its first row
  auto first_qt = [&](int kt) { return PASS == kLse ? un.qt : kt * kRows <= sq.q0 ? 0 : (kt * kRows - sq.q0) / kRows; };
  auto end_qt = [&]() { return PASS == kLse ? un.qt + 1 : nqt; };
  bool ok = true;

  if (warp == kSWarps) {
    // ---------------- loads ----------------
    if (lane == 0) {
      const int row0 = (int)((int64_t)a.layer * a.H * a.C) + sq.row0 + h * sq.cap;
      uint32_t nk = 0, nq = 0;
      for (int kt = un.kt0; ok && kt < un.kt1; ++kt, ++nk) {
        const int st = nk % KS;
        if (nk >= KS && !(ok = pf_wait(&k_empty[st], (nk / KS & 1) ^ 1, limit_ns))) break;
        mbar_arrive_expect_tx(&k_full[st], Cf::TILE);
#pragma unroll
        for (int i = 0; i < Cf::NSUB; ++i)
          tma_load_2d(sm + st * Cf::TILE + i * Cf::SUBB, &mk, i * Cf::SUB, row0 + kt * kRows, &k_full[st]);
        for (int qt = first_qt(kt); qt < end_qt(); ++qt) {
          if (PASS != kSumMany && nq > 0) break;  // one query tile, which stays
          const int qs = nq % QS;
          if (nq >= QS && !(ok = pf_wait(&q_empty[qs], (nq / QS & 1) ^ 1, limit_ns))) break;
          mbar_arrive_expect_tx(&q_full[qs], Cf::QT);
          const uint32_t dst = sm + Cf::Q_OFF + qs * Cf::QT;
#pragma unroll
          for (int i = 0; i < Cf::NSUB; ++i) {
            const int x = i * Cf::SUB, z = sq.tok0 + qt * kRows;
            tma_load_3d(dst + i * Cf::QSUBB, &mq, x, h, z, &q_full[qs]);
            if constexpr (NQ > 1) tma_load_3d(dst + Cf::QTILE + i * Cf::QSUBB, &mq1, x, h, z, &q_full[qs]);
            if constexpr (NQ > 2) tma_load_3d(dst + 2 * Cf::QTILE + i * Cf::QSUBB, &mq2, x, h, z, &q_full[qs]);
          }
          ++nq;
        }
      }
      // never leave with copies in flight (every full barrier's last phase)
      for (int i = 0; i < KS; ++i)
        if ((uint32_t)i < nk) (void)pf_wait(&k_full[i], ((nk - 1 - i) / KS) & 1, limit_ns);
      for (int i = 0; i < QS; ++i)
        if ((uint32_t)i < nq) (void)pf_wait(&q_full[i], ((nq - 1 - i) / QS) & 1, limit_ns);
    }
    __syncwarp();
  } else if (warp == kSWarps + 1) {
    // ---------------- products ----------------
    // columns: the keys, or the queries, where there is one tile of them no more than there are (64 of 128: the second pass
    // of the window of 64 has half the work)
    const int n_col = PASS == kLse || PASS == kSumMany ? kRows : (sq.len - sq.q0 + 15) & ~15;
    const uint32_t id = mma_idesc(Pack16<T>::kType, 0, kRows, n_col);
    constexpr uint32_t SBO = 8 * Cf::SW;
    auto uni_wait = [&](uint64_t* bar, uint32_t parity) -> bool { return __all_sync(0xFFFFFFFFu, pf_wait(bar, parity, limit_ns)); };
    uint32_t nk = 0, nq = 0, step = 0;
    for (int kt = un.kt0; ok && kt < un.kt1; ++kt, ++nk) {
      const int st = nk % KS;
      if (!(ok = uni_wait(&k_full[st], nk / KS & 1))) break;
      const uint32_t k_d = desc_lo(sm + st * Cf::TILE, 16);
      const int qe = end_qt();
      for (int qt = first_qt(kt); qt < qe; ++qt, ++step) {
        const int qs = PASS == kSumMany ? nq % QS : 0, sb = step & 1;
        if ((PASS == kSumMany || nq == 0) && !(ok = uni_wait(&q_full[qs], nq / QS & 1))) break;
        if (step >= 2 && !(ok = uni_wait(&s_empty[sb], (step / 2 & 1) ^ 1))) break;
        tc_fence_after();
        const uint32_t q_d = desc_lo(sm + Cf::Q_OFF + qs * Cf::QT, 16);
        if (elect_one()) {
#pragma unroll
          for (int part = NQ - 1; part >= 0; --part) {  // the small parts first: the tensor core cuts what it adds to a sum
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = ((kk * 16) / Cf::SUB * Cf::SUBB + (kk * 16) % Cf::SUB * 2) >> 4;
              const uint32_t qoff = ((kk * 16) / Cf::SUB * Cf::QSUBB + (kk * 16) % Cf::SUB * 2) >> 4;
              const uint64_t dk = desc(k_d + off, SBO, Cf::SW), dq = desc(q_d + part * (Cf::QTILE >> 4) + qoff, SBO, Cf::SW);
              tc_mma(tmem + sb * kRows, PASS == kLse ? dq : dk, PASS == kLse ? dk : dq, id, part < NQ - 1 || kk > 0);
            }
          }
          tc_commit(&s_full[sb]);
          if (PASS == kSumMany) tc_commit(&q_empty[qs]);
          if (qt + 1 == qe) tc_commit(&k_empty[st]);
        }
        __syncwarp();
        ++nq;
      }
    }
  } else {
    // ---------------- S ----------------
    const int half = warp >> 2;
    const int r = (warp & 3) * 32 + lane;  // the thread's row of S (its TMEM lane)
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const float2 cc = make_float2(a.c2, a.c2);
    constexpr int NC = QN < 64 ? QN : 64;  // columns taken at a time
    float s[NC];
    auto s_wait = [&](uint32_t step) -> bool {
      const bool got = __all_sync(0xFFFFFFFFu, pf_wait(&s_full[step & 1], step / 2 & 1, limit_ns));
      tc_fence_after();
      return got;
    };
    // columns [c, c + NC) of the step's S into registers
    auto take = [&](uint32_t step, int c) {
      if constexpr (NC == 64) {
        tmem_ld32(lanes + (step & 1) * kRows + c, s);
        tmem_ld32(lanes + (step & 1) * kRows + c + 32, s + 32);
      } else {
        tmem_ld16(lanes + (step & 1) * kRows + c, s);
      }
      tmem_wait_ld();
    };
    auto s_done = [&](uint32_t step) {
      tc_fence_before();
      mbar_arrive(&s_empty[step & 1]);
    };
    // the columns whose bit is missing
    auto hide = [&](uint32_t v0, uint32_t v1) {
      if (__all_sync(0xFFFFFFFFu, (v0 & v1) == 0xFFFFFFFFu)) return;
#pragma unroll
      for (int x = 0; x < NC; ++x)
        if (!((x < 32 ? v0 : v1) >> (x & 31) & 1)) s[x] = -INFINITY;
    };
    // The steps of the passes over key tiles go to the halves by turns (a half's steps all have the same buffer of S).
    [[maybe_unused]] auto mine = [&](uint32_t step) { return (int)(step & 1) == half; };
    if constexpr (PASS == kLse) {
      const int t0 = sq.q0 + un.qt * kRows, t1 = min(t0 + kRows, sq.len), t = t0 + r;  // the query's stored row
      const bool live = t < sq.len;
      const bool idle = t0 + (warp & 3) * 32 >= sq.len;  // none of the warp's queries exists
      const bool is_cl = live && (a.meta[sq.moff + t] & 1);
      // a <CL> query's sum is its own row's: the half that has this row begins anew there, the last that it sees
      const bool mine_cl = is_cl && (t >> 6 & 1) == half && t / kRows >= un.kt0 && t / kRows < un.kt1;
      float m = -INFINITY, l = 0.f;
      for (int kt = un.kt0; kt < un.kt1; ++kt) {
        const int i0 = kt * kRows + half * 64;  // the row of the thread's first column
        uint32_t v0 = 0xFFFFFFFFu, v1 = v0;
        if (a.least[sq.moff / kRows + kt] < t1 - 1) {  // a row of the tile is hidden from some of the queries
          const int h0 = __ldg(a.meta + sq.moff + i0 + lane) >> 1, h1 = __ldg(a.meta + sq.moff + i0 + 32 + lane) >> 1;
          v0 = ~__ballot_sync(0xFFFFFFFFu, h0 < t0);
          v1 = ~__ballot_sync(0xFFFFFFFFu, h1 < t0);
          // rows that some of the queries see and others do not: spans that end among the queries
          for (uint32_t p = __ballot_sync(0xFFFFFFFFu, h0 >= t0 && h0 < t1 - 1); p; p &= p - 1) {
            const int x = __ffs(p) - 1;
            if (t > __shfl_sync(0xFFFFFFFFu, h0, x)) v0 &= ~(1u << x);
          }
          for (uint32_t p = __ballot_sync(0xFFFFFFFFu, h1 >= t0 && h1 < t1 - 1); p; p &= p - 1) {
            const int x = __ffs(p) - 1;
            if (t > __shfl_sync(0xFFFFFFFFu, h1, x)) v1 &= ~(1u << x);
          }
        }
        if (i0 + 63 > t0) {  // later rows
          v0 &= low_bits(t - i0 + 1);
          v1 &= low_bits(t - i0 - 31);
          if (mine_cl && (uint32_t)(t - i0) < 64u) {
            v0 = low_bits(t - i0 + 1) & ~low_bits(t - i0);
            v1 = low_bits(t - i0 - 31) & ~low_bits(t - i0 - 32);
            m = -INFINITY;
            l = 0.f;
          }
        }
        const uint32_t step = kt - un.kt0;
        if (!(ok = s_wait(step))) break;
        take(step, half * 64);
        s_done(step);
        if (idle || !__any_sync(0xFFFFFFFFu, v0 | v1)) continue;
        hide(v0, v1);
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int x = 4; x < 64; x += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = fmaxf(mx[e], s[x + e]);
        const float mn = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.c2), mu = mn == -INFINITY ? 0.f : mn;
        float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
        const float2 mm = make_float2(-mu, -mu);
#pragma unroll
        for (int x = 0; x < 64; x += 4) {
          const float2 z0 = __ffma2_rn(make_float2(s[x], s[x + 1]), cc, mm);
          const float2 z1 = __ffma2_rn(make_float2(s[x + 2], s[x + 3]), cc, mm);
          sum0 = __fadd2_rn(sum0, make_float2(ex2(z0.x), ex2(z0.y)));
          sum1 = __fadd2_rn(sum1, make_float2(ex2(z1.x), ex2(z1.y)));
        }
        l = l * ex2(m - mu) + ((sum0.x + sum0.y) + (sum1.x + sum1.y));
        m = mn;
      }
      if (is_cl && !mine_cl) {
        m = -INFINITY;
        l = 0.f;
      }
      if (half) s_half[r] = make_float2(m, l);
      bar_sync(1, kSThreads);
      if (!half && ok && live) {
        const float2 o = s_half[r];
        const float M = fmaxf(m, o.x), Mu = M == -INFINITY ? 0.f : M;
        a.lse[((int64_t)un.split * a.H + h) * a.n_tok + sq.tok0 + un.qt * kRows + r] =
            make_float2(M, l * ex2(m - Mu) + o.y * ex2(o.x - Mu));
      }
    } else if constexpr (PASS == kLse16) {
      // A key per thread: each keeps the maximum and sum of every query over its own keys, joined at the end.
      float m[QN], l[QN];
#pragma unroll
      for (int x = 0; x < QN; ++x) {
        m[x] = -INFINITY;
        l[x] = 0.f;
      }
      // the <CL> queries, which see their own rows alone
      const uint32_t cl = __ballot_sync(0xFFFFFFFFu, lane < sq.len - sq.q0 && (a.meta[sq.moff + min(sq.q0 + lane, sq.len - 1)] & 1));
      for (int kt = un.kt0; kt < un.kt1; ++kt) {
        const uint32_t step = kt - un.kt0;
        if (!mine(step)) continue;
        const int i = kt * kRows + r, hid = i < sq.len ? a.meta[sq.moff + i] >> 1 : -1;
        const int lo = max(i - sq.q0, 0), hi = min(hid, sq.len - 1) - sq.q0;
        const uint32_t others = cl & ~(low_bits(i - sq.q0 + 1) & ~low_bits(i - sq.q0));
        if (!(ok = s_wait(step))) break;
        take(step, 0);
        s_done(step);
        hide((low_bits(hi + 1) & ~low_bits(lo) & ~others) | ~low_bits(QN), 0xFFFFFFFFu);
#pragma unroll
        for (int x = 0; x < QN; ++x) {
          const float z = s[x] * a.c2, mn = fmaxf(m[x], z), mu = mn == -INFINITY ? 0.f : mn;
          l[x] = l[x] * ex2(m[x] - mu) + ex2(z - mu);
          m[x] = mn;
        }
      }
#pragma unroll
      for (int x = 0; x < QN; ++x) {
        float M = m[x];
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, off));
        float L = l[x] * ex2(m[x] - (M == -INFINITY ? 0.f : M));
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, off);
        if (lane == x) s_half[warp * QN + x] = make_float2(M, L);
      }
      bar_sync(1, kSThreads);
      if (tid < sq.len - sq.q0 && ok) {
        float M = -INFINITY, L = 0.f;
        for (int w = 0; w < kSWarps; ++w) {
          const float2 v = s_half[w * QN + tid];
          const float Mn = fmaxf(M, v.x), Mu = Mn == -INFINITY ? 0.f : Mn;
          L = L * ex2(M - Mu) + v.y * ex2(v.x - Mu);
          M = Mn;
        }
        a.lse[((int64_t)un.split * a.H + h) * a.n_tok + sq.tok0 + tid] = make_float2(M, L);
      }
    } else {
      // -L of query tile qt's r-th query; -infinity for none, NaN where its weights are not numbers: a logit is NaN or
      // +infinity, or all are -infinity
      auto neg_lse = [&](int qt) -> float {
        const int x = qt * kRows + r;
        if (sq.q0 + x >= sq.len) return -INFINITY;
        const float2* p = a.lse + (int64_t)h * a.n_tok + sq.tok0 + x;
        const int64_t step_s = (int64_t)a.H * a.n_tok;
        float M = -INFINITY, L = 0.f;
        for (int k = 0; k < a.n_split; ++k) {
          const float2 v = __ldcg(p + k * step_s);
          const float Mn = fmaxf(M, v.x), Mu = Mn == -INFINITY ? 0.f : Mn;
          L = L * ex2(M - Mu) + v.y * ex2(v.x - Mu);
          M = Mn;
        }
        const float lse = M + log2f(L);
        return fabsf(lse) < INFINITY ? -lse : NAN;
      };
      pdl_wait();  // the queries' sums
      auto cl_query = [&](int qt) -> bool {  // and whether it is a <CL>
        const int t = sq.q0 + qt * kRows + r;
        return t < sq.len && (a.meta[sq.moff + t] & 1);
      };
      auto load_neg = [&](float neg, bool is_cl) {  // for the half's next step; its threads are done with the last one's
        bar_sync(1 + half, kSThreads / 2);
        // such a query's weight is NaN at the rows that it sees, and must not reach the others of its columns
        s_neg[half][r] = neg == neg ? neg : -INFINITY;
        const uint32_t bad = __ballot_sync(0xFFFFFFFFu, neg != neg), none = __ballot_sync(0xFFFFFFFFu, neg == -INFINITY);
        const uint32_t cl = __ballot_sync(0xFFFFFFFFu, is_cl);
        if (lane == 0) {
          s_none[half][warp & 3] = none | bad | cl;
          s_bad[half][warp & 3] = bad;
          s_cl[half][warp & 3] = cl;
        }
        bar_sync(1 + half, kSThreads / 2);
      };
      if (PASS == kSumFew) load_neg(neg_lse(0), cl_query(0));
      uint32_t step = 0;
      for (int kt = un.kt0; kt < un.kt1; ++kt) {
        const int i = kt * kRows + r;
        const bool row = i < sq.len;
        const int meta = row ? a.meta[sq.moff + i] : 0, hid = meta >> 1;
        float total = 0.f;
        bool any = false;  // the half had a step of this key tile
        [[maybe_unused]] float next = 0.f;
        [[maybe_unused]] bool next_cl = false;
        const int qe = end_qt();
        for (int qt = first_qt(kt); qt < qe; ++qt, ++step) {
          if (!mine(step)) continue;
          if (PASS == kSumMany) {
            load_neg(any ? next : neg_lse(qt), any ? next_cl : cl_query(qt));
            if (qt + 2 < qe) {
              next = neg_lse(qt + 2);
              next_cl = cl_query(qt + 2);
            }
          }
          any = true;
          const int t0 = sq.q0 + qt * kRows, t1 = min(t0 + kRows, sq.len);
          // after a wait that ran out the warp only keeps up with the others' barriers
          if (!ok || !(ok = s_wait(step))) continue;
          const int lo = max(i - t0, 0), hi = row ? min(hid, t1 - 1) - t0 : -1;  // the columns that see row i
          const uint4 bad = *reinterpret_cast<const uint4*>(s_bad[half]);
          if (bad.x | bad.y | bad.z | bad.w) {
            const uint32_t b[4] = {bad.x, bad.y, bad.z, bad.w};
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (b[c] & low_bits(hi + 1 - 32 * c) & ~low_bits(lo - 32 * c) & ~s_cl[half][c]) total = NAN;
          }
          if ((meta & 1) && i >= t0 && i < t1)  // a <CL> query's weight is its own row's: 1, whatever its logit, if that is finite
            total += s_bad[half][(i - t0) >> 5] >> ((i - t0) & 31) & 1 ? NAN : 1.f;
#pragma unroll 1
          for (int c = 0; c < QN; c += NC) {
            const uint32_t v0 = low_bits(hi + 1 - c) & ~low_bits(lo - c) & ~s_none[half][c / 32];
            const uint32_t v1 = low_bits(hi - 31 - c) & ~low_bits(lo - 32 - c) & ~s_none[half][(c / 32 + 1) & 3];
            const bool seen = __any_sync(0xFFFFFFFFu, v0 | v1);
            if (seen) take(step, c);
            if (c + NC == QN) s_done(step);
            if (!seen) continue;
            hide(NC == 64 ? v0 : v0 | ~low_bits(NC), NC == 64 ? v1 : 0xFFFFFFFFu);
            const float4* neg = reinterpret_cast<const float4*>(s_neg[half] + c);
            float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
#pragma unroll
            for (int x = 0; x < NC; x += 4) {
              const float4 n = neg[x / 4];
              const float2 z0 = __ffma2_rn(make_float2(s[x], s[x + 1]), cc, make_float2(n.x, n.y));
              const float2 z1 = __ffma2_rn(make_float2(s[x + 2], s[x + 3]), cc, make_float2(n.z, n.w));
              sum0 = __fadd2_rn(sum0, make_float2(ex2(z0.x), ex2(z0.y)));
              sum1 = __fadd2_rn(sum1, make_float2(ex2(z1.x), ex2(z1.y)));
            }
            total += (sum0.x + sum0.y) + (sum1.x + sum1.y);
          }
        }
        if (PASS == kSumMany) {  // a key tile's steps are of both halves: the first adds them up
          if (half) s_half[r].x = total;
          bar_sync(3, kSThreads);
          if (!half) total += s_half[r].x;
          any = !half;
        }
        if (any && ok && row) {
          float* sc = a.scores + ((int64_t)a.layer * a.H * a.C + sq.row0 + (int64_t)h * sq.cap + i);
          *sc += total;
        }
        if (PASS == kSumMany && kt + 1 < un.kt1) bar_sync(3, kSThreads);  // s_half is read
      }
    }
  }
  if (!ok) atomicOr(a.status, STATUS_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256u) : "memory");
  }
}

// The queries of a 128-query tile (blockIdx.x), rotated at their positions, in parts.
template <typename T, int D>
__global__ void __launch_bounds__(256) score_rotate_kernel(const ScoreArgs a) {
  constexpr int CH = D / 8, NQ = kFullParts<T>;
  const ScoreUnit un = a.units[blockIdx.x];
  if (un.split != 0) return;
  const ScoreSeq& sq = un.q;
  const int n = min(kRows, sq.len - sq.q0 - un.qt * kRows);
  for (int x = blockIdx.y * 256 + threadIdx.x; x < n * a.H * CH; x += gridDim.y * 256) {
    const int r = x / (a.H * CH), w = x - r * (a.H * CH), c = w % CH;
    const int64_t row = ((int64_t)(sq.tok0 + un.qt * kRows + r) * a.H + w / CH) * D;
    uint32_t part[NQ][4];
    query_chunk<T, NQ>(a.q + row, c, a.rot, a.pos[a.off[sq.s] + sq.q0 + un.qt * kRows + r], a.rope_g, part);
#pragma unroll
    for (int i = 0; i < NQ; ++i)
      *reinterpret_cast<uint4*>(a.q_part + i * a.part_stride + row + c * 8) = make_uint4(part[i][0], part[i][1], part[i][2], part[i][3]);
  }
}

template <typename T, int D, int NQ, int PASS, int QN>
cudaError_t launch_score_t(const ScoreMaps& maps, const ScoreArgs& a, cudaStream_t stream) {
  using Cf = ScCfg<D, NQ, PASS, QN>;
  static std::atomic<bool> done[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!done[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(score_kernel<T, D, NQ, PASS, QN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cf::SMEM);
    if (e != cudaSuccess) return e;
    done[dev].store(true, std::memory_order_release);
  }
  CUtensorMap mk, mq[3];
  std::memcpy(&mk, maps.k, sizeof mk);
  for (int i = 0; i < 3; ++i) std::memcpy(&mq[i], maps.q[i < NQ ? i : 0], sizeof mq[i]);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((int64_t)a.n_units * a.H));
  cfg.blockDim = dim3(kScThreads);
  cfg.dynamicSmemBytes = Cf::SMEM;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PASS == kLse || PASS == kLse16 ? 0 : 1;  // the first pass starts when all before it is complete
  return cudaLaunchKernelEx(&cfg, score_kernel<T, D, NQ, PASS, QN>, mk, mq[0], mq[1], mq[2], a);
}

template <typename F>
cudaError_t by_type(const Geometry& g, F&& f) {
  auto dt = [&](auto dc) { return g.dtype == 1 ? f(BF16T{}, dc) : f(F16T{}, dc); };
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

template <int PASS, int QN>
cudaError_t launch_pass(const Geometry& g, const ScoreMaps& maps, const ScoreArgs& a, cudaStream_t stream) {
  if (a.n_units <= 0) return cudaSuccess;
  return by_type(g, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return g.rot > 0 ? launch_score_t<T, D, kFullParts<T>, PASS, QN>(maps, a, stream)
                     : launch_score_t<T, D, 1, PASS, QN>(maps, a, stream);
  });
}

}  // namespace

int score_parts(const Geometry& g) { return g.rot == 0 ? 1 : g.dtype == 1 ? kFullParts<BF16T> : kFullParts<F16T>; }

int score_ctas_per_sm(const Geometry& g) {
  int n = 1;
  (void)by_type(g, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    n = g.rot > 0 ? ScCfg<D, kFullParts<T>, kLse, kRows>::CPS : ScCfg<D, 1, kLse, kRows>::CPS;
    return cudaSuccess;
  });
  return n;
}

cudaError_t launch_score_rotate(const Geometry& g, const ScoreArgs& a, cudaStream_t stream) {
  if (a.n_units <= 0) return cudaSuccess;
  return by_type(g, [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    score_rotate_kernel<T, D><<<dim3((unsigned)a.n_units, 16), 256, 0, stream>>>(a);
    return cudaGetLastError();
  });
}

cudaError_t launch_score_lse(const Geometry& g, const ScoreMaps& maps, const ScoreArgs& a, int most, cudaStream_t stream) {
  return most <= 16 ? launch_pass<kLse16, 16>(g, maps, a, stream) : launch_pass<kLse, kRows>(g, maps, a, stream);
}

cudaError_t launch_score_sum(const Geometry& g, const ScoreMaps& maps, const ScoreArgs& a, int most, cudaStream_t stream) {
  return most <= 16      ? launch_pass<kSumFew, 16>(g, maps, a, stream)
         : most <= kRows ? launch_pass<kSumFew, kRows>(g, maps, a, stream)
                         : launch_pass<kSumMany, kRows>(g, maps, a, stream);
}

}  // namespace kvc
