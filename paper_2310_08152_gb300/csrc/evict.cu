// Eviction by accumulated attention weight: every (layer, head) stream of a sequence keeps its recent rows and, of the
// others, those whose scores are largest.
//
// A stream of n rows keeps `keep`, the last `recent` of them whatever their scores.  Of its n - recent candidates the
// A = keep - recent with the largest scores stay (ties: the lower row; a NaN counts below every number).  Attention does
// not depend on the order of the rows, so as few as possible move: the candidates that stay and lie below row A stay
// where they are, the j-th row below A that goes is replaced by the j-th candidate beyond it that stays, and the recent
// rows, whose order the span bookkeeping relies on, move down behind them.
//
// One CTA, or a cluster where there are few streams, per stream:
//   1. the A-th largest score by radix selection (11 + 11 + 10 bits of the scores' ordered bit patterns, kept in shared
//      memory), stopping at the first digit whose bin stays whole;
//   2. two scans in row order, over the rows below A and over those beyond, list the holes and the rows that fill them;
//      the copies of one list's rows are disjoint from each other, so they need no barrier between them;
//   3. the recent rows move down through shared memory with 1-D bulk copies: the first chunk is under way from the
//      kernel's start, while the scores are sorted (moved by registers after that, the step of 12,288 streams that drop
//      one of 1,025 rows took 231 us), and goes back once the holes are filled; the rest follow chunk by chunk.
// What bounds it: HBM, for the rows that move, and for evictions of few rows the selection, some barriers per stream.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "device_common.cuh"
#include "kernels.hpp"

namespace kvc {
namespace {

constexpr unsigned kFull = 0xFFFFFFFFu;
constexpr int kBins = 2048;
constexpr int kMaxHeldKeys = 40 * 1024;  // candidates whose keys stay in shared memory (160 KB); else they are read again
constexpr int kMaxCluster = 8;
constexpr int kFewDrops = 4;  // rows that go, at most, for which the least score is looked for row by row

// A score's order as an unsigned number: a NaN below everything, -0 and +0 equal.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ void bulk_s2g(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_addr(src)), "r"(bytes)
               : "memory");
}

template <int kThreads>
struct EvictShared {
  static constexpr int kWarps = kThreads / 32;
  static constexpr int kScan = 4 * kThreads;  // candidates of one scan step
  union {
    uint32_t hist[kBins];
    struct {
      int32_t holes[kScan], srcs[2 * kScan];
    } l;
  };
  uint64_t full;
  uint64_t least[2][kWarps];
  int32_t dropped[kFewDrops];
  uint32_t wsum[kWarps];
  uint32_t bin, above, in_bin;
};

// Exclusive prefix of one value per thread over the block, and the block's sum (two barriers).
template <int kThreads>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, EvictShared<kThreads>& sh, uint32_t* sum) {
  constexpr int kWarps = kThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t u = __shfl_up_sync(kFull, incl, d);
    if (lane >= d) incl += u;
  }
  if (lane == 31) sh.wsum[warp] = incl;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const uint32_t x = sh.wsum[w];
    before += w < warp ? x : 0u;
    all += x;
  }
  __syncthreads();
  *sum = all;
  return before + incl - v;
}

// IMG: the call's upload is a parameter (of img_bytes, its AffSeqs from aff_off on), which the first CTA stores at dyn.
struct NoImage {};
template <int D, int kThreads, bool IMG>
__global__ void __launch_bounds__(kThreads, kThreads == 128 ? 7 : 1024 / kThreads)
    evict_kernel(Geometry g, Static st, Buffers buf, float* __restrict__ scores, const AffSeq* __restrict__ aff_,
                 int32_t* __restrict__ kept, int held, int chunk, int CN,
                 const __grid_constant__ std::conditional_t<IMG, AppendImage, NoImage> img, int img_bytes, int aff_off,
                 uint4* __restrict__ dyn_out) {
  constexpr int VPR = D / 8;  // 16-byte vectors per row
  const AffSeq* aff = aff_;
  if constexpr (IMG) {
    aff = reinterpret_cast<const AffSeq*>(reinterpret_cast<const unsigned char*>(&img) + aff_off);
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i < (img_bytes + 15) / 16; i += kThreads) dyn_out[i] = img.v[i];
  }
  extern __shared__ __align__(128) unsigned char dyn[];
  // `chunk` recent rows of K and then of V (of one of them in a cluster), then the keys
  uint32_t* keys = reinterpret_cast<uint32_t*>(dyn + (size_t)chunk * (CN > 1 ? 1 : 2) * D * 2);
  __shared__ EvictShared<kThreads> sh;
  constexpr int kWarps = EvictShared<kThreads>::kWarps, kScan = EvictShared<kThreads>::kScan;
  const int tid = threadIdx.x;
  const int rank = CN > 1 ? (int)(blockIdx.x % (unsigned)CN) : 0;
  const int unit = CN > 1 ? (int)(blockIdx.x / (unsigned)CN) : (int)blockIdx.x;
  const int streams = g.M * g.H;
  const AffSeq a = aff[unit / streams];
  const int sidx = unit % streams, m = sidx / g.H, h = sidx % g.H;
  const int n = a.len_old, keep = a.len_new, recent = a.first_row;
  const int A = keep - recent, cand = n - recent;
  const int64_t row0 = (int64_t)m * g.H * g.C + st.seq_row0[a.s] + (int64_t)h * st.cap[a.s];
  float* sc = scores + row0;
  int32_t* kp = kept ? kept + row0 : nullptr;
  uint4* K = reinterpret_cast<uint4*>(buf.k + row0 * D);
  uint4* V = reinterpret_cast<uint4*>(buf.v + row0 * D);
  const bool in_smem = cand <= held;
  // Recent rows [r, min(r + chunk, recent)) into shared memory; the first two of a cluster's CTAs take K and V.
  const bool do_k = CN == 1 || (rank & 1) == 0, do_v = CN == 1 || (rank & 1) == 1;
  auto load_recent = [&](int r) {
    const uint32_t bytes = (uint32_t)min(chunk, recent - r) * D * 2;
    mbar_arrive_expect_tx(&sh.full, bytes * (CN > 1 ? 1 : 2));
    if (do_k) bulk_g2s(dyn, K + (int64_t)(cand + r) * VPR, bytes, &sh.full);
    if (do_v) bulk_g2s(dyn + (CN > 1 ? 0 : (size_t)chunk * D * 2), V + (int64_t)(cand + r) * VPR, bytes, &sh.full);
  };
  if (tid == 0) {
    mbar_init(&sh.full, 1);
    fence_mbar_init();
    if (rank < 2) load_recent(0);
  }
  auto key = [&](int i) { return in_smem ? keys[i] : order_key(sc[i]); };

  // Moves the rows of the first n_hole entries of the lists.
  auto move = [&](int n_hole) {
    constexpr int U = kThreads == 128 ? 2 : 4;
    const int step = CN * kThreads, total = n_hole * VPR;
    for (int v0 = rank * kThreads + tid; v0 < total; v0 += U * step) {
      uint4 k[U], v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = v0 + u * step;
        if (x < total) {
          const int64_t at = (int64_t)sh.l.srcs[x / VPR] * VPR + x % VPR;
          k[u] = K[at];
          v[u] = V[at];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = v0 + u * step;
        if (x < total) {
          const int64_t at = (int64_t)sh.l.holes[x / VPR] * VPR + x % VPR;
          K[at] = k[u];
          V[at] = v[u];
        }
      }
    }
    if (rank == 0)
      for (int j = tid; j < n_hole; j += kThreads) {
        const int to = sh.l.holes[j], from = sh.l.srcs[j];
        sc[to] = sc[from];
        if (kp != nullptr) kp[to] = from;
      }
  };
  const int drop = cand - A;
  if (A > 0 && drop <= kFewDrops && in_smem) {
    // A few rows go (every step of a generation at its budget): the least score, of equal ones the highest row's, is found
    // and taken out `drop` times, two barriers each, instead of the selection's and the scans' thirty (the step of 12,288
    // streams that drop one of 1,025 rows: 223 us with those).
    for (int i = tid; i < cand; i += kThreads) keys[i] = order_key(sc[i]);
    for (int d = 0; d < drop; ++d) {
      uint64_t best = ~0ull;
      for (int i = tid; i < cand; i += kThreads) best = min(best, (uint64_t)keys[i] << 32 | (0xFFFFFFFFu - (uint32_t)i));
#pragma unroll
      for (int off = 16; off >= 1; off >>= 1) best = min(best, __shfl_xor_sync(kFull, best, off));
      if ((tid & 31) == 0) sh.least[d & 1][tid >> 5] = best;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kWarps; ++w) best = min(best, sh.least[d & 1][w]);
      const int row = (int)(0xFFFFFFFFu - (uint32_t)best);
      if (row % kThreads == tid) keys[row] = 0xFFFFFFFFu;  // above every score's key; the thread that reads it
      if (tid == 0) sh.dropped[d] = row;
    }
    if (rank == 0 && kp != nullptr)
      for (int i = tid; i < A; i += kThreads) kp[i] = i;
    __syncthreads();
    int n_hole = 0;
    for (int d = 0; d < drop; ++d) n_hole += sh.dropped[d] < A;
    if (tid < drop) {
      const int row = sh.dropped[tid];
      int below = 0;  // dropped rows below it
      for (int d = 0; d < drop; ++d) below += sh.dropped[d] < row;
      if (row < A) sh.l.holes[below] = row;
      // rows A .. A + drop - 1 that stay: the tid-th of them, less the dropped ones below it
      const int src = A + tid;
      bool stays = true;
      int rank_src = tid;
      for (int d = 0; d < drop; ++d) {
        stays = stays && sh.dropped[d] != src;
        rank_src -= sh.dropped[d] >= A && sh.dropped[d] < src;
      }
      if (stays) sh.l.srcs[rank_src] = src;
    }
    __syncthreads();
    if (CN > 1) cluster_sync();  // every CTA of the cluster has read the scores
    move(n_hole);
  } else {
    // ------------------------------ the A-th largest score ---------------------------------------
    uint32_t T = 0;              // stays: key > T, and the first `need` (in row order) with key == T
    int need = 0x7FFFFFFF;
    bool ties = false;           // fewer of the equal ones stay than there are
    if (A > 0) {
      if (in_smem)
        for (int i = tid; i < cand; i += kThreads) keys[i] = order_key(sc[i]);
      uint32_t prefix = 0, want = (uint32_t)A;
      int shift = 21;
      for (int pass = 0; pass < 3; ++pass) {
        const int width = pass == 2 ? 10 : 11;
        const int hi = shift + width;  // the digits above are `prefix`
#pragma unroll
        for (int b = 0; b < kBins / kThreads; ++b) sh.hist[b * kThreads + tid] = 0;
        __syncthreads();
        const uint32_t mask = (1u << width) - 1u;
        for (int i = tid; i < cand; i += kThreads) {
          const uint32_t k = key(i);
          if (pass == 0 || k >> hi == prefix) atomicAdd(&sh.hist[(k >> shift) & mask], 1u);
        }
        __syncthreads();
        // thread t holds the t-th `per` bins from the top down
        const int per = kBins / kThreads, top = kBins - 1 - tid * per;
        uint32_t c[kBins / kThreads], mine = 0;
#pragma unroll
        for (int b = 0; b < per; ++b) {
          c[b] = sh.hist[top - b];
          mine += c[b];
        }
        uint32_t all;
        uint32_t above = block_scan(mine, sh, &all);
        if (above < want && want <= above + mine) {
#pragma unroll
          for (int b = 0; b < per; ++b) {
            if (above < want && want <= above + c[b]) {
              sh.bin = (uint32_t)(top - b);
              sh.above = above;
              sh.in_bin = c[b];
            }
            above += c[b];
          }
        }
        __syncthreads();
        prefix = prefix << width | sh.bin;
        want -= sh.above;
        T = prefix << shift;
        if (want == sh.in_bin) break;  // the whole bin stays: every key from its lowest on
        if (pass == 2) {
          need = (int)want;
          ties = true;
        }
        shift -= pass == 1 ? 10 : 11;
        __syncthreads();
      }
      // no key of the bin's range lies at or below T but T itself, so "key >= T" is "key > T or the equal ones"
    }

    // ------------------------------ holes, and the rows that fill them ---------------------------
    const uint32_t uneed = (uint32_t)need;
    uint32_t eq_hole = 0, eq_src = 0;  // equal ones before each scan's next candidate
    if (ties) {                        // those below row A
      uint32_t c = 0;
      for (int i = tid; i < A; i += kThreads) c += key(i) == T;
      block_scan(c, sh, &eq_src);
    }
    __syncthreads();
    if (CN > 1) cluster_sync();  // every CTA of the cluster has read the scores
    // One step of a scan: the candidates [base, min(base + kScan, end)) that stay (or go) are appended to list at *count.
    auto scan = [&](int base, int end, uint32_t& eq_before, bool stay, int32_t* list, int count) {
      uint32_t gt = 0, eq = 0;
      const int i0 = base + 4 * tid;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + u < end) {
          const uint32_t k = key(i0 + u);
          gt |= (uint32_t)(k > T) << u;
          eq |= (uint32_t)(k == T) << u;
        }
      }
      uint32_t sum;
      const uint32_t pre = block_scan(__popc(gt) | __popc(eq) << 16, sh, &sum);
      uint32_t e = eq_before + (pre >> 16);
      uint32_t stayed = (pre & 0xFFFFu) + (min(e, uneed) - min(eq_before, uneed));
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u;
        if (i < end) {
          const bool s = (gt >> u & 1u) || ((eq >> u & 1u) && e < uneed);
          e += eq >> u & 1u;
          if (stay && s) list[count + stayed] = i;
          if (!stay && !s) list[count + (uint32_t)(i - base) - stayed] = i;
          if (!stay && s && kp != nullptr && rank == 0) kp[i] = i;
          stayed += s;
        }
      }
      const int total = (int)((sum & 0xFFFFu) + (min(eq_before + (sum >> 16), uneed) - min(eq_before, uneed)));
      eq_before += sum >> 16;
      __syncthreads();
      return stay ? total : min(end - base, kScan) - total;
    };
    int at_src = A, n_src = 0;
    for (int at_hole = 0; at_hole < A; at_hole += kScan) {
      const int n_hole = scan(at_hole, A, eq_hole, false, sh.l.holes, 0);
      while (n_src < n_hole && at_src < cand) {
        n_src += scan(at_src, cand, eq_src, true, sh.l.srcs, n_src);
        at_src += kScan;
      }
      if (n_hole > n_src) {  // cannot be: as many stay beyond row A as go below it
        if (tid == 0) atomicOr(buf.status, STATUS_CHECK);
        break;
      }
      move(n_hole);
      __syncthreads();
      // the rows not used yet go to the front of their list
      const int left = n_src - n_hole;
      int32_t keep_src[kScan / kThreads];
#pragma unroll
      for (int u = 0; u < kScan / kThreads; ++u) {
        const int j = u * kThreads + tid;
        if (j < left) keep_src[u] = sh.l.srcs[n_hole + j];
      }
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kScan / kThreads; ++u) {
        const int j = u * kThreads + tid;
        if (j < left) sh.l.srcs[j] = keep_src[u];
      }
      n_src = left;
      __syncthreads();
    }
  }
  if (CN > 1)
    cluster_sync();
  else
    __syncthreads();

  // ------------------------------ the recent rows move down ------------------------------------
  // Rows move down, so a chunk's places lie below every later chunk's rows.
  if (tid == 0 && rank < 2) {
    bool ok = true;
    int phase = 0;
    for (int r = 0; r < recent; r += chunk, phase ^= 1) {
      if (r > 0) {
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the last chunk is read
        load_recent(r);
      }
      if (!(ok = mbar_wait_bounded(&sh.full, phase, 2000000000ull))) break;
      const uint32_t bytes = (uint32_t)min(chunk, recent - r) * D * 2;
      if (do_k) bulk_s2g(K + (int64_t)(A + r) * VPR, dyn, bytes);
      if (do_v) bulk_s2g(V + (int64_t)(A + r) * VPR, dyn + (CN > 1 ? 0 : (size_t)chunk * D * 2), bytes);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    if (!ok) {
      atomicOr(buf.status, STATUS_TIMEOUT);
      (void)mbar_wait_bounded(&sh.full, phase, 2000000000ull);  // never leave with a copy in flight
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if (rank == 0) {
    const bool meta = m == 0 && h == 0;  // the sequence's positions and history indices
    int32_t* pos = buf.pos + st.off[a.s];
    int32_t* orig = buf.orig + st.off[a.s];
    for (int i0 = 0; i0 < recent; i0 += kThreads) {
      const int i = i0 + tid;
      const bool in = i < recent;
      const float s = in ? sc[cand + i] : 0.f;
      const int32_t po = in && meta ? pos[cand + i] : 0, oo = in && meta ? orig[cand + i] : 0;
      __syncthreads();
      if (in) {
        sc[A + i] = s;
        if (kp != nullptr) kp[A + i] = cand + i;
        if (meta) {
          pos[A + i] = po;
          orig[A + i] = oo;
        }
      }
    }
    __syncthreads();
    for (int i = keep + tid; i < n; i += kThreads) sc[i] = 0.f;
    if (meta)
      for (int i = tid; i < A; i += kThreads) pos[i] = orig[i] = -1;  // they differ between streams now
  }
}

template <int D, int NT, bool IMG>
cudaError_t launch_evict_t(const Geometry& g, const Static& st, const Buffers& buf, float* scores, const AffSeq* aff,
                           int n_aff, int64_t max_cand, int64_t max_recent, int32_t* kept, int num_sms,
                           const EvictImage* image, cudaStream_t stream) {
  static std::atomic<bool> done[64];
  constexpr int kMost = 200 * 1024;  // of dynamic shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!done[dev].load(std::memory_order_acquire)) {
    e = cudaFuncSetAttribute(evict_kernel<D, NT, IMG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
    done[dev].store(true, std::memory_order_release);
  }
  const int64_t units = (int64_t)n_aff * g.M * g.H;
  // keys that do not fit are read again from the scores, which the CTAs of a cluster would change under each other
  const int held = (int)std::min<int64_t>(max_cand, kMaxHeldKeys);
  int cn = 1;
  if (max_cand <= kMaxHeldKeys)
    while (2 * cn <= kMaxCluster && 2 * cn * units <= 2 * num_sms) cn *= 2;
  // recent rows of a chunk: 16 KB of K and V, which leaves room for seven CTAs of 128 threads per SM, or 24 KB
  const int chunk = (int)std::min<int64_t>(max_recent, (cn > 1 ? 2 : 1) * (NT == 128 ? 8 : 12) * 1024 / (D * 2));
  const size_t smem = (size_t)chunk * (cn > 1 ? 1 : 2) * D * 2 + 4 * (size_t)held;
  static_assert(32 * 1024 + 4 * kMaxHeldKeys <= kMost, "shared memory");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * cn));
  cfg.blockDim = dim3(NT);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cn;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cn > 1 ? 1 : 0;
  if constexpr (IMG)
    return cudaLaunchKernelEx(&cfg, evict_kernel<D, NT, IMG>, g, st, buf, scores, aff, kept, held, chunk, cn, *image->img,
                              image->bytes, image->aff_off, static_cast<uint4*>(image->dyn));
  else
    return cudaLaunchKernelEx(&cfg, evict_kernel<D, NT, IMG>, g, st, buf, scores, aff, kept, held, chunk, cn, NoImage{}, 0, 0,
                              static_cast<uint4*>(nullptr));
}

}  // namespace

cudaError_t launch_evict(const Geometry& g, const Static& st, const Buffers& buf, float* scores, const AffSeq* aff,
                         int n_aff, int64_t max_cand, int64_t max_recent, int64_t max_drop, int32_t* kept,
                         int num_sms, const EvictImage* image, cudaStream_t stream) {
  if (n_aff <= 0) return cudaSuccess;
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    // Threads by the candidates, where more than a few go.  us with 128 / 256 / 512 threads: 12,288 streams of 960, 64 of
    // them, 244 / 264 / -; 2,048 of 1,592, 256 of them, 129 / 119 / 141; 1,024 of 1,984, 1,536 of them, 77 / 55 / 62;
    // 1,024 of 4,436, 500 of them, 149 / 127 / 115.  A few: 12,288 of 897, one of them, 147 / 174 / -.
    auto by = [&](auto nt) {
      constexpr int NT = decltype(nt)::value;
      return image != nullptr ? launch_evict_t<D, NT, true>(g, st, buf, scores, aff, n_aff, max_cand, max_recent, kept,
                                                            num_sms, image, stream)
                              : launch_evict_t<D, NT, false>(g, st, buf, scores, aff, n_aff, max_cand, max_recent, kept,
                                                             num_sms, image, stream);
    };
    if (max_drop <= kFewDrops || max_cand <= 1280) return by(std::integral_constant<int, 128>{});
    return max_cand <= 3000 ? by(std::integral_constant<int, 256>{}) : by(std::integral_constant<int, 512>{});
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
