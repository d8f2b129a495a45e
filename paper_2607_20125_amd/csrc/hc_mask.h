// The mask with a window and first tokens, and the pages of a cache, on the device.
// Included by the .hip sources only.
#pragma once

#include "hc_seq.h"

namespace hc {
namespace dev {

// Keys that a query sees: [0, sink) and [start, end).  All three grow with the query.
struct Seen {
  int end, sink, start;
  // (without branches: a mask asks for many keys)
  __device__ __forceinline__ bool sees(int key) const { return (key < end) & ((key < sink) | (key >= start)); }
};
// Query i of n over m keys.  (32 bits without a sign hold the end of any position's block.)
__device__ __forceinline__ Seen seen_of(int block, int window, int sinks, int n, int m, int i) {
  if (block == 0) return {m, 0, 0};
  const int p = m - n + i;
  if (p < 0) return {0, 0, 0};
  const uint32_t end = ((uint32_t)p / (uint32_t)block + 1) * (uint32_t)block;
  Seen s;
  s.end = (int)min(end, (uint32_t)m);
  s.start = window == 0 || end <= (uint32_t)window ? 0 : (int)min(end - (uint32_t)window, (uint32_t)s.end);
  s.sink = min(sinks, s.start);
  return s;
}
__device__ __forceinline__ Seen seen_by(const SeqArgs &a, const SeqUnit &u, int i) {
  return seen_of(a.block, a.window, a.sinks, u.nq, u.nk, i);
}

// Key tiles that any row of a unit sees, counted without the gap between the first tokens and the window:
// tile t is at place(t) of the sequence.
struct KeyTiles {
  int n;                     // tiles
  int first, gap;            // tiles of the first tokens; tiles left out behind them
  int lo_start, lo_end, hi_sink, hi_start, hi_end;      // of the first and last query
  __device__ __forceinline__ KeyTiles(Seen lo, Seen hi) {
    first = (hi.sink + kSeqKeys - 1) / kSeqKeys;
    gap = max(lo.start / kSeqKeys - first, 0);
    n = (hi.end + kSeqKeys - 1) / kSeqKeys;
    if (n <= first + gap) gap = max(n - first, 0);      // (the window begins where the keys end)
    n -= gap;
    lo_start = lo.start;
    lo_end = lo.end;
    hi_sink = hi.sink;
    hi_start = hi.start;
    hi_end = hi.end;
  }
  __device__ __forceinline__ int place(int t) const { return t + (t >= first ? gap : 0); }
  // Whether every row sees all of the tile at this place.
  __device__ __forceinline__ bool whole(int at, int sinks) const {
    return (at + 1) * kSeqKeys <= lo_end && ((at + 1) * kSeqKeys <= sinks || at * kSeqKeys >= hi_start);
  }
};

// The four runs of 16 keys of a tile, in pages: lane l reads the entry of run l % 4.  (A page holds
// whole runs.  Runs behind the last key take the last key's.)
__device__ __forceinline__ int run_of(const SeqUnit &u, int at, int j) { return min(at * 4 + j, (u.nk - 1) >> 4); }
__device__ __forceinline__ int page_entry(const SeqArgs &a, const SeqUnit &u, int at, int lane) {
  return a.table[(int64_t)u.seq * a.table_seq + (int)(((int64_t)run_of(u, at, lane & 3) << 4) >> a.page_shift)];
}
// Bit j: run j has no page.
__device__ __forceinline__ uint32_t absent_runs(const SeqArgs &a, int entry) {
  return (uint32_t)__ballot((uint32_t)entry >= (uint32_t)a.n_pages) & 15u;
}
// The page of run j (page 0 for one that is absent: nothing of it counts).
__device__ __forceinline__ int page_of(const SeqArgs &a, int entry, int j) {
  const int p = __builtin_amdgcn_readlane(entry, j);
  return (uint32_t)p < (uint32_t)a.n_pages ? p : 0;
}
// First token of a run in its page.
__device__ __forceinline__ int run_token(const SeqArgs &a, int run) { return (run << 4) & ((1 << a.page_shift) - 1); }

constexpr float kLn2 = 0.6931471805599453f;
// The logarithm of a row's sum of exponentials from its maximum and sum in log2 units.
__device__ __forceinline__ float log_sum(float m, float l) {
  return l > 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : l == 0.f ? -INFINITY : l;
}

}  // namespace dev
}  // namespace hc
