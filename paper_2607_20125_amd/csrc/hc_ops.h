// Internal structures of the operators beside the routed attention (hc_ops.cpp,
// hc_rotate.hip, hc_qcache.hip, hc_seq.hip, hc_seq128.hip, hc_decode.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "headcast.h"

namespace hc {

// --- rotary positions -----------------------------------------------------------
constexpr int kRotMaxDim = 256, kRotMaxAxes = 4;

struct RotateArgs {
  hc_rotate_tensor t[2];
  const int32_t *positions;      // [n_axes][n_tokens], or null: from the grid
  int32_t n_tokens, head_dim, rot;
  int32_t n_axes, axis_end[kRotMaxAxes];   // first pair behind each axis
  int32_t grid_h, grid_w, frame0;
  int32_t heads;                 // of both tensors
  int32_t heads_per;             // heads that one thread takes
  int32_t items;                 // threads per token
  float sign;                    // of the angle
  double turns[kRotMaxDim / 2];  // angle per position step of each pair, in turns
};
hipError_t launch_rotate(const RotateArgs &a, int x_type, int out_type, bool halves, hipStream_t s);

// --- the 4-bit cache --------------------------------------------------------------
// A sequence's head is a run of 64-token tiles, each one contiguous:
//   K codes  [64 tokens][d / 2 bytes]
//   K scales [64 tokens][d / 32]
//   V codes  [8 groups of 8 tokens][d / 4][8 tokens][2 bytes: 4 dims]
//   V scales [8 groups][d / 32][8 tokens]
// A scale is the biased exponent of its power of two, 255 for a group that is not
// finite; a byte holds two codes, the lower dim in its low half.  V is grouped by 8
// tokens because the product with the probabilities needs 8 keys of one dim side by
// side: 16 bytes hold 4 dims of such a group.  A tile (8.5 KB for 128 dims) is what a
// wave or work group reads in one go.
constexpr int kQTokens = 64, kQGroup = 32;
constexpr int kScaleLow = 2, kScaleHigh = 252, kScaleNone = 255;   // biased exponents
constexpr int qtile_k_scales(int d) { return kQTokens * d / 2; }
constexpr int qtile_v(int d) { return kQTokens * (d / 2 + d / kQGroup); }
constexpr int qtile_v_scales(int d) { return qtile_v(d) + kQTokens * d / 2; }
constexpr int qtile_bytes(int d) { return 2 * qtile_v(d); }
inline __host__ __device__ int64_t qcache_head_bytes(int capacity, int d) {
  return ((int64_t)capacity + kQTokens - 1) / kQTokens * qtile_bytes(d);
}

struct QCacheArgs {
  hc_qcache cache;
  hc_qcache_rows rows;
};
hipError_t launch_qcache_append(const QCacheArgs &a, hipStream_t s);
hipError_t launch_qcache_read(const QCacheArgs &a, hipStream_t s);

// --- attention over sequences -------------------------------------------------------
// The rows of a (sequence, key head) are its queries times the query heads of that key
// head: row r is query r / group, head r % group.  A unit is a run of kSeqRows of them
// (kDecodeRows in the kernel for few rows), and units may be cut into key ranges whose
// partial results a second launch merges.
constexpr int kSeqRows = 128, kDecodeRows = 16, kSeqKeys = 64;
constexpr int kSeqMaxSplit = 32, kDecodeMaxSplit = 256;
struct SeqArgs {
  const uint16_t *q;
  uint16_t *o;
  int64_t q_token, q_head, o_token, o_head;
  const uint16_t *k, *v;         // packed keys and values, or null: the cache
  int64_t k_token, k_head, v_token, v_head;
  const uint8_t *cache;
  int64_t cache_head;            // bytes per head; a sequence has kv_heads of them
  int32_t capacity;
  const int32_t *cu_q, *cu_k, *kv_len;
  int32_t n_seqs, n_tokens, n_keys;
  int32_t kv_heads, group;
  int32_t block;                 // 0: every key is seen
  int32_t tiles;                 // units of a key head that the launch has room for
  // Units, numbered tile * kv_heads + head: the first `whole` are one work group each, the others are cut
  // into n_split key ranges, whose work groups come after those.
  int32_t whole, n_split;
  int32_t *head;                 // cut units: [unit - whole][4]: q0, row0, rows (0: no such unit)
  float *part;                   // [unit - whole][n_split][seq_part_floats]
  float scale_log2;              // softmax scale * log2(e)
  bool wide;                     // 128-dim heads: waves of 64 rows (hc_seq128.hip)
  // attention with a window (hc_window.cpp)
  int32_t window, sinks;         // window 0: every earlier key
  float *lse;                    // [heads][n_tokens], or null
  // the cache in pages: k and v are page 0, `capacity` slots a sequence
  const int32_t *table;
  int64_t table_seq, k_page, v_page;
  int32_t n_pages, page_shift;
};
inline int64_t seq_units(const SeqArgs &a) { return (int64_t)a.tiles * a.kv_heads; }
inline int64_t seq_cut_units(const SeqArgs &a) { return a.n_split > 1 ? seq_units(a) - a.whole : 0; }
inline int64_t seq_groups(const SeqArgs &a) { return a.whole + (seq_units(a) - a.whole) * a.n_split; }
// Floats of one partial result: rows of d sums, then the rows' maxima and sums, and where logarithms are asked for the
// sums of the probabilities before their rounding.
constexpr int64_t seq_part_floats(int rows, int d, bool logs = false) { return (int64_t)rows * (d + (logs ? 3 : 2)); }
hipError_t launch_seq(const SeqArgs &a, int head_dim, hipStream_t s);
hipError_t launch_seq128(const SeqArgs &a, hipStream_t s);
hipError_t launch_decode(const SeqArgs &a, int head_dim, hipStream_t s);
hipError_t launch_seq_merge(const SeqArgs &a, int head_dim, int rows, hipStream_t s);

}  // namespace hc
