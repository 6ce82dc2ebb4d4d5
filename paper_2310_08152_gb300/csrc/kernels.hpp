// Internal interface between the host state (kvc.cpp) and the sm_103a kernels (kernels.cu).
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

namespace kvc {

// Per-sequence decode state, uploaded after every change of the span book.
// The decode query of sequence s reads stored rows [begin, len) except [mask_lo, mask_hi).  Row
// begin + r lives in slot begin + r while r < wrap and in slot r - wrap after it (a ring, for the
// local-attention cache; wrap is INT32_MAX otherwise).
struct DState {
  int32_t len, begin, mask_lo, mask_hi, qpos, wrap;
  int32_t is_cl;  // a <CL> query: it sees its own row only, and none of a prefix
  int32_t pad;
};

// One stored token: its sequence, destination row, position, history index, and its index among
// the input tokens of the call (tokens freed as they are written have no plan entry).
struct TokPlan {
  int32_t s, row, pos, orig, in_tok, pad0, pad1, pad2;
};

// One sequence of a compaction, or of an eviction (see launch_evict); its drop ranges (history indices, [lo, hi)) are
// ranges[range_off .. range_off + n_ranges).
struct AffSeq {
  int32_t s, len_old, len_new, first_row, range_off, n_ranges, pad0, pad1;
};

// Status word bits written by kernels.
enum : int { STATUS_TIMEOUT = 1, STATUS_CHECK = 2 };

struct Geometry {
  int M, H, D, b;
  int64_t C;  // sum of capacities (rows per (layer, K/V, head) plane)
  int dtype;  // 0 f16, 1 bf16
  int rot;    // rotary dims (0 = none)
};

struct Static {
  const int64_t* seq_row0;  // [b] H * off[s]
  const int32_t* cap;       // [b]
  const int64_t* off;       // [b]
  const float2* rope_g;     // [rot/2] theta_i / (2 pi) per position as a double-float (hi, lo)
};

struct Buffers {
  uint16_t* k;   // cache K base
  uint16_t* v;   // cache V base
  int32_t* pos;  // [C]
  int32_t* orig; // [C]
  int* status;
};

// Most decode workers (warps); sizes the split-K partial buffer.
constexpr int kMaxDecodeWorkers = 8192;

bool dhead_supported(int D);

// The planes of a cache of 4 bits (packed.cuh): [M][H * C] rows of D / 2 bytes of codes and of packed_groups(D) words of
// (lo, step) pairs, for K and for V.  Its sequences' capacities in the layout are multiples of kPackedRows, so that a run
// of rows that starts at a multiple of it starts at 16 bytes in every plane.
struct PackedBuffers {
  unsigned char* kc;
  unsigned char* vc;
  uint32_t* kp;
  uint32_t* vp;
};
constexpr int kPackedRows = 4;
inline int packed_groups(int D) { return (D + 31) / 32; }
// The decode's work is counted in tiles of kPackedTile rows, from row begin / kPackedRows * kPackedRows of a segment on, and
// kPackedPiece more for each segment: P then holds the prefix sums of that.  Each worker (warp) has a counter and two parts of
// D + 4 floats.
constexpr int kPackedTile = 64, kPackedPiece = 1;
constexpr int kMaxPackedWorkers = 4096;

// Writes the n_plan stored tokens of a call whose inputs hold n_in tokens per layer (k_in, v_in
// 16-byte aligned).  maps: the device copy of encode_append_maps' output, or NULL; with it, calls of
// at least num_sms (layer, token) units go through the TMA kernel, whose bounded waits give up
// after limit_ns.
cudaError_t launch_append(const Geometry& g, const Static& st, const Buffers& buf, const TokPlan* plan, int64_t n_plan,
                          int64_t n_in, int m0, int n_layers, bool write_meta, const void* k_in, const void* v_in,
                          const void* maps, int num_sms, unsigned long long limit_ns, cudaStream_t stream);
// Of all layers or of layer 0, for uploads (img_bytes, a multiple of 16, the plan from plan_off on) that fit a kernel
// parameter; they go to dyn.
struct alignas(16) AppendImage {
  uint4 v[224];
};
cudaError_t launch_append_image(const Geometry& g, const Static& st, const Buffers& buf, const AppendImage& img,
                                size_t img_bytes, size_t plan_off, void* dyn, int64_t n_plan, int64_t n_in,
                                int n_layers, const void* k_in, const void* v_in, cudaStream_t stream);
// The same of a cache of 4 bits: K is rotated and rounded as above, then packed.  img: the upload as a kernel parameter
// (img_bytes, the plan from plan_off on, stored at dyn), or NULL and the plan on the device.
cudaError_t launch_packed_append(const Geometry& g, const Static& st, const Buffers& buf, const PackedBuffers& pb,
                                 const TokPlan* plan, const AppendImage* img, size_t img_bytes, size_t plan_off, void* dyn,
                                 int64_t n_plan, int64_t n_in, int m0, int n_layers, bool write_meta, const void* k_in,
                                 const void* v_in, cudaStream_t stream);
// Bytes of encode_append_maps' output: a 128-byte TMA descriptor per (K/V, sequence).
inline size_t append_maps_bytes(int b) { return 2 * 128 * (size_t)b; }
// Encodes, per sequence s, 4-D TMA descriptors over the K and then the V planes: dims {D, cap[s],
// H, M} from row seq_row0[s] of layer 0's plane, strides (D, cap[s] D, H C D) elements, box
// {D, 1, H, 1}: one (layer, token)'s rows of every head.  seq_row0 and cap are host arrays; out is
// host memory of append_maps_bytes(b).  cudaErrorNotSupported where a box cannot hold H heads.
cudaError_t encode_append_maps(const Geometry& g, const Buffers& buf, const int64_t* seq_row0, const int32_t* cap,
                               unsigned char* out);

// Scan, then row moves.  between: an event recorded on the stream between the two kernels, or NULL.  packed: the planes of
// a cache of 4 bits, whose rows are moved instead of buf's.
cudaError_t launch_compact(const Geometry& g, const Static& st, const Buffers& buf, const AffSeq* aff, int n_aff,
                           const int32_t* ranges, int32_t* src_map, cudaStream_t stream, int* launched,
                           cudaEvent_t between = nullptr, const PackedBuffers* packed = nullptr);
cudaError_t launch_packed_move(const Geometry& g, const Static& st, const PackedBuffers& pb, const AffSeq* aff, int n_aff,
                               const int32_t* src_map, cudaStream_t stream);

struct DecodeArgs {
  int device;            // the current device
  int layer;             // the first layer of the launch
  int n_layers = 1;      // layers layer .. layer + n_layers - 1 in one launch (whole segments only)
  const DState* dstate;  // [b]
  const int64_t* P;      // [b+1] prefix sums of attended-range lengths (len - begin)
  int64_t R;             // H * P[b]
  const void* q;         // [b][H][D] per layer, layer i at q + i * q_layer_stride elements
  float* out;            // [b][H][D] per layer, layer i at out + i * out_layer_stride floats
  int64_t q_layer_stride = 0;
  int64_t out_layer_stride = 0;
  float scale;
  float* partials;       // [(kMaxDecodeWorkers + b*H) * (D + 4)]
  int* counters;         // [b*H], zero between launches
  unsigned long long wait_limit_ns;
  // 1 when the kernel launched before this one on the stream was a decode (which writes no K/V):
  // K/V tiles are then requested before that kernel has completed (programmatic dependent launch).
  int kv_before_wait;
  // segment statistics of the uploaded state: segments with rows, and the longest one
  int64_t n_segments;
  int64_t max_segment;
};

// How a decode launch split its work: mode 0 = unbalanced segments of one layer, a CTA or cluster per
// (sequence, head) segment or stream-K over all rows; 1 = balanced segments, a CTA or cluster each or
// up to eight per CTA; 2 = one warp per segment; 3 = several consecutive whole segments per warp;
// 4 = unbalanced segments over several layers, one or two per CTA or runs of whole segments per warp
// cut by rows; workers = warps that attend; tile rows; stages.
struct DecodePlan {
  int mode, workers, tile_rows, stages;
};

// Returns the grid used through *grid (0 if nothing launched) and the plan through *plan.  A launch
// over several layers (a.n_layers > 1) takes whole segments only: where unbalanced segments are fewer
// than a wave of CTAs, or the longest too long beside the rest, it launches nothing and returns
// cudaErrorNotSupported, and the caller goes layer by layer.
cudaError_t launch_decode(const Geometry& g, const Static& st, const Buffers& buf, const DecodeArgs& a,
                          int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan);

// The decode of a cache of 4 bits, all the launch's layers together (a.P and a.R as above; a.counters:
// [kMaxPackedWorkers], zero between launches).
cudaError_t launch_packed_decode(const Geometry& g, const Static& st, const PackedBuffers& pb, const DecodeArgs& a,
                                 int* status, int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan);

// The decode with each row's attention weight added to its score (scores: [M][H * C], in the rows' layout): a CTA or a
// cluster per segment, or several segments per CTA, whatever the segments.
cudaError_t launch_decode_scored(const Geometry& g, const Static& st, const Buffers& buf, const DecodeArgs& a,
                                 float* scores, int num_sms, cudaStream_t stream, int* grid, DecodePlan* plan);

// The prefix part of a shared-prefix decode (prefix.cu).  A unit is a run of a prefix's rows for some of its members.
struct PrefixUnit {
  int32_t s;           // sequence of the prefix's cache
  int32_t key0, key1;  // its stored rows
  int32_t mem0, n_mem; // members[mem0 ..], as many as a CTA takes at most
  int32_t split;       // the run's number among the prefix's
  int32_t pad0, pad1;
};
struct PrefixArgs {
  int layer, n_layers, H, rot;
  int64_t C;                // of the prefix's cache, as st, k and v
  Static st;
  const uint16_t* k;
  const uint16_t* v;
  const PrefixUnit* units;  // [n_units], for each (layer, head)
  int n_units;
  const int32_t* members;   // sequences of the own rows' cache
  const DState* ds;         // theirs
  // sequence s has n_split[s] parts, from entry split0[s] on; entry e of head h in the launch's layer i starts at
  // parts + ((i * n_parts + e) * H + h) * (D + 4) floats: maximum and sum (exp2 domain), two unused, then D columns
  const int32_t* split0;
  const int32_t* n_split;
  int64_t n_parts;
  float* parts;
  const uint16_t* q;        // [b][H][D] per layer, 16-byte aligned
  int64_t q_stride;
  float c2;                 // scale * log2(e)
  int* status;
  unsigned long long wait_limit_ns;
};
// The own rows' part, joined with the prefix's.
struct OwnArgs {
  PrefixArgs px;            // st, k, v, C of the own rows' cache here
  int b;
  float* out;               // [b][H][D] per layer
  int64_t out_stride;
  // The kernel before this one is the prefix kernel, of less than a wave: this one may start beside it and waits before it
  // reads the parts.  Beside a larger one its waiting CTAs take room from it (8 samples of 8 prefixes of 800 rows, 32
  // layers: 646 us, one after the other 588).
  int early;
  float* scores = nullptr;  // launch_own_scored: as launch_decode_scored's
};
// The scored decode of many short segments (n_segments of all layers, `rows` rows in all) by the same kernel, without a
// prefix; whether it is the one for them.
bool own_scored_takes(int64_t n_segments, int64_t rows, int64_t max_segment, int num_sms);
cudaError_t launch_own_scored(const Geometry& g, const OwnArgs& a, cudaStream_t stream, DecodePlan* plan);
// Queries of one CTA (16 or 32: launch_prefix; kPrefixTcRows: launch_prefix_tc, with maps of the prefix's planes): as many
// as the largest group of `group` members may need, or fewer in several CTAs, where most groups are small.  What a row
// costs a CTA of so many queries, in twentieths of a row of 16 queries: all prefixes of one length, us with 16 / 32 / 128
// queries: 16 groups of 8 and one of 33, d_head 80, f16, 548 / 828 / 833, d_head 128, bf16, 387 / 583 / 461; 8 of 8 and 8 of
// 64 1321 / 1464 / 1214 and 707 / 835 / 466; 16 of 33 1437 / 1712 / 1178 and 842 / 1033 / 457; 4 of 8 and 4 of 40 501 / 641 /
// 515 and 330 / 447 / 246.
constexpr int kPrefixTcRows = 128;
int prefix_rows(int group);
inline int prefix_row_cost(int rows, int d_head) { return rows == 16 ? 20 : rows == 32 ? 31 : d_head == 128 ? 27 : 36; }
// CTAs per SM of that kernel.
cudaError_t prefix_ctas_per_sm(const Geometry& g, int device, int rows, int* occ);
cudaError_t launch_prefix(const Geometry& g, const PrefixArgs& a, int device, int rows, cudaStream_t stream);
struct alignas(64) PrefixMaps {
  unsigned char k[128], v[128];
};
cudaError_t launch_prefix_tc(const Geometry& g, const PrefixMaps& maps, const PrefixArgs& a, cudaStream_t stream);

cudaError_t launch_own(const Geometry& g, const OwnArgs& a, int64_t max_segment, int num_sms, cudaStream_t stream,
                       DecodePlan* plan);

// Scores follow their rows through a compaction (after launch_compact, from the same source map): in place, zero in
// the slots that lost their row.
cudaError_t launch_compact_scores(const Geometry& g, const Static& st, float* scores, const AffSeq* aff, int n_aff,
                                  const int32_t* src_map, cudaStream_t stream);

// Eviction (evict.cu): in every (layer, head) stream of the n_aff sequences, len_new of len_old rows stay, the last
// `first_row` of them (the recent ones) and those with the largest scores.  max_cand, max_recent, max_drop: the most
// candidates, recent rows and rows that go of a stream; kept: [M][H * C] or NULL, the earlier row number of each kept row.
// image: the call's upload (state and AffSeqs) as a kernel parameter, where it fits one, stored at dyn by the kernel
// (an eviction of two sequences in two layers: an upload and its event less, 23 us of host time before); else NULL.
struct EvictImage {
  const AppendImage* img;
  int bytes, aff_off;
  void* dyn;
};
cudaError_t launch_evict(const Geometry& g, const Static& st, const Buffers& buf, float* scores, const AffSeq* aff,
                         int n_aff, int64_t max_cand, int64_t max_recent, int64_t max_drop, int32_t* kept,
                         int num_sms, const EvictImage* image, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------
// Masked prefill attention (prefill.cu)
// ---------------------------------------------------------------------------------------------
// A prefill query tile as the host lays it out: queries [qr0, qr_end) (stored rows) of sequence s, the
// first of them token tok0 of the q / out arrays; a work item is one tile of one head.  Its keys
// are the stored rows some query of the tile may see, in order: the first n_c rows of the sequence's list
// of rows that no span hides (klist[moff ..]; below vb they are the stored rows of the same number), then
// stored rows [b0, qr0) -- the interior of a span that begins before the tile and ends in it or after it,
// if there is one (else b0 = qr0) --, then the tile's own rows; nk tiles of keys.  The per-row mask bounds
// start at meta[moff]; row0 = seq_row0[s], the K/V plane row of stored row 0 of head 0 in layer 0 (the
// kernel adds layer * H * C + h * cap).
struct PfTileRec {
  int32_t n_c, b0, tok0, moff;
  int32_t s, cap, qr0, qr_end;
  int32_t nk, row0, vb, pad;
};
static_assert(sizeof(PfTileRec) == 48, "three 16-byte loads");
// The work items in the kernel's order.
struct PfItemRec {
  int32_t tile, h;
};

struct PrefillArgs {
  int layer, H, rot;
  int64_t C;
  const PfItemRec* items;  // [n_items]: sequences with the most stored rows first, then head, then the query tile with the most keys first
  const PfTileRec* tiles;  // [n_items / H]: in the same order, without the heads
  int64_t n_items;         // (query tile, head) work items
  unsigned long long* item_counter;  // [2], zero at launch and after it: the next item, the CTAs that are through
  int n_ctas;              // persistent grid size
  const int32_t* meta;     // per stored row: (hid << 1) | is_cl
  const int32_t* klist;    // per sequence, from the same offset as meta: the stored rows no span hides
  const uint16_t* k;       // the K and V planes of every layer
  const uint16_t* v;
  const uint16_t* q;       // [sum n_q][H][D]
  float* out;              // [sum n_q][H][D]
  int64_t n_qtok;          // sum n_q
  float c2;                // scale * log2(e)
  const int32_t* pos;      // [C] stored-row positions
  const int64_t* off;      // [b]: a sequence's first entry in pos
  const float2* rope_g;    // [rot/2]
  int* status;
  unsigned long long wait_limit_ns;
};

// Encoded 2-D TMA descriptors of the K and V planes ([M*H*C rows][D], swizzled column subtiles).
struct alignas(64) PrefillMaps {
  unsigned char k[128];
  unsigned char v[128];
  bool ready = false;
};

cudaError_t encode_prefill_maps(const Geometry& g, const Buffers& buf, PrefillMaps* maps);
// A 2-D map of the K or the V planes (base) as above in boxes of 128 rows; a 3-D map of queries [n_tok][H][D] in boxes of one column
// subtile x one head x `rows` tokens.  out: 128 bytes.
cudaError_t encode_rows_map(const Geometry& g, const void* base, unsigned char* out);
cudaError_t encode_query_map(const Geometry& g, const void* q, int64_t n_tok, int rows, unsigned char* out);
// Most CTAs of the persistent prefill grid.
constexpr int kMaxPrefillCtas = 1024;
// Keys of one key tile for head dimension D and the cache type, and where a tile's own rows start among
// its keys when n_before come before them: on a key tile of their own when those divide a query tile.
int prefill_keys_per_tile(int D, int dtype);
inline int prefill_own_start(int n_before, int kt) { return 128 % kt == 0 ? (n_before + kt - 1) / kt * kt : n_before; }
// CTAs of the prefill kernel that fit on one SM for head dimension D (sizes the persistent grid).
int prefill_ctas_per_sm(int D);
// A persistent grid of a.n_ctas CTAs walks the a.n_items work items.
cudaError_t launch_prefill(const Geometry& g, const PrefillMaps& maps, const PrefillArgs& a, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------
// Scores of a prompt (score.cu)
// ---------------------------------------------------------------------------------------------
// A sequence with queries: they are stored rows [q0, len), tokens tok0 .. of q; row0 = seq_row0[s]; its rows' mask bounds
// (as the prefill's) start at meta[moff], a multiple of 128, the least `hid` of each 128 rows at least[moff / 128].
struct alignas(16) ScoreSeq {
  int32_t tok0, q0, len, moff, row0, cap, s, pad;
};
// A unit of the first pass: key tiles [kt0, kt1) for query tile qt; of the second: key tiles [kt0, kt1).
struct alignas(16) ScoreUnit {
  ScoreSeq q;
  int32_t qt, kt0, kt1, split;
};
struct ScoreArgs {
  int layer, H, rot;
  int64_t C, n_tok;         // tokens of q
  const ScoreUnit* units;   // of the pass
  int n_units;              // each for H heads
  const int32_t* meta;
  const int32_t* least;
  float2* lse;              // [n_split][H][n_tok]: (maximum, sum) of each query over a split's keys, exp2 domain
  int n_split;
  float* scores;            // [M][H * C]
  float c2;
  int* status;
  unsigned long long wait_limit_ns;
  // rotated queries: their 16-bit parts, part_stride elements apart
  const uint16_t* q;
  uint16_t* q_part;
  int64_t part_stride;
  const int32_t* pos;
  const int64_t* off;
  const float2* rope_g;
};
struct alignas(64) ScoreMaps {
  unsigned char k[128], q[3][128];
};
// 16-bit parts that the queries go as: one, or of rotated ones two (f16) or three (bf16).
int score_parts(const Geometry& g);
// Resident CTAs per SM of the passes' kernels (sizes the units).
int score_ctas_per_sm(const Geometry& g);
// Rotates a.q into a.q_part, the query tile of each of the first pass's units with split 0 (the others' blocks end at once).
cudaError_t launch_score_rotate(const Geometry& g, const ScoreArgs& a, cudaStream_t stream);
// The passes; most: the most queries of a sequence.  The boxes of the query maps hold score_query_rows(most) tokens.
inline int score_query_rows(int most) { return most <= 16 ? 16 : 128; }
cudaError_t launch_score_lse(const Geometry& g, const ScoreMaps& maps, const ScoreArgs& a, int most, cudaStream_t stream);
cudaError_t launch_score_sum(const Geometry& g, const ScoreMaps& maps, const ScoreArgs& a, int most, cudaStream_t stream);

// ---------------------------------------------------------------------------------------------
// Copies of sequences (copy.cu)
// ---------------------------------------------------------------------------------------------
// A source sequence and its targets: targets[first .. first + n); its rows are chunks chunk0 .. of the call's.
struct alignas(16) CopySource {
  int32_t s, len, first, n, chunk0, pad0, pad1, pad2;
};
// Rows of a chunk, which a block copies: 16 KB of 16-bit rows of 64 columns, and twice as many that become 4-bit ones.
constexpr int copy_rows(int dst_bits) { return dst_bits == 4 ? 256 : 128; }
// A target sequence, the rows that it held before, the rows that it holds now, and the source sequence.
struct alignas(16) CopyTarget {
  int32_t s, len_old, len, src;
};
// One side of a copy: planes of 16 bits (bits 16: k, v) or of 4.
struct CopySide {
  int bits;
  int64_t C;
  Static st;
  uint16_t* k;
  uint16_t* v;
  PackedBuffers pb;
  int32_t* pos;
  int32_t* orig;
  float* scores;  // or NULL
};
// img: the targets' upload (decode state, sources, targets) as a kernel parameter, stored at dyn, or NULL.  sources and
// targets: offsets in that upload.  n_chunks: of all sources.
struct CopyArgs {
  CopySide src, dst;
  int n_sources, n_targets;
  int64_t n_chunks;
  size_t sources, targets;
  const AppendImage* img;
  size_t img_bytes;
  void* dyn;
};
// The blocks that the kernels take, which have to be at most INT32_MAX.
inline int64_t copy_blocks(const Geometry& g, const CopyArgs& a) {
  return std::max(a.n_chunks * g.M * 2 * g.H, a.dst.scores ? (int64_t)a.n_targets * g.M * g.H : 1);
}
// Rows and metadata; then, where the targets' cache has scores, theirs (the source's or zero, and zero behind them).
cudaError_t launch_copy(const Geometry& g, const CopyArgs& a, cudaStream_t stream, int* launched);
// Stores an upload that comes as a kernel parameter, and zeroes the scores of rows [len, len_old) of the targets in it.
cudaError_t launch_drop(const Geometry& g, const CopyArgs& a, cudaStream_t stream, int* launched);

// One warp waits on an mbarrier phase that never completes, with the limit given; the bounded wait
// gives up and sets STATUS_TIMEOUT in *status.  Exercises the kernels' timeout reporting.
cudaError_t launch_bounded_wait_check(int* status, unsigned long long limit_ns, cudaStream_t stream);

// Split-K scratch in a file-scope device array (kernels.cu), for callers that cannot allocate
// device memory.  *ptr gets its device address on the current device; the address is looked up
// with cudaGetSymbolAddress the first time a device asks for it.
constexpr size_t kStaticDecodeScratchBytes = size_t(8) << 20;
cudaError_t static_decode_scratch(void** ptr);

}  // namespace kvc
