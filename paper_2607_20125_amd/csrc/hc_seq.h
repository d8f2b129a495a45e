// Device-side helpers of the attention over sequences and of the 4-bit cache.
// Included by the .hip sources only.
#pragma once

#include "hc_device.h"
#include "hc_ops.h"

namespace hc {
namespace dev {

// Two stored values, byte B of a word of codes, in bf16 (exact: two bits of
// significand).  A scale of infinity (the mark of a group that is not finite) gives NaN.
template <int B>
__device__ __forceinline__ uint32_t values2(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}

// Byte B of a word of scale codes as its power of two.
template <int B>
__device__ __forceinline__ float scale_of(uint32_t codes) {
  return __uint_as_float((codes >> (8 * B) & 0xffu) << 23);
}

// One unit of work: rows row0 .. of a sequence (row r is query r / group).
struct SeqUnit {
  int seq;
  int row0, rows;          // first row, rows of the sequence
  int nq, nk;
  int64_t q0, k0;          // first query and key of the sequence in the packed tensors
};

// Unit `tile` of the launch, in units of R rows; false if there is none.  Called by
// whole waves.  Later units of a sequence come first: with a causal mask they have the most keys,
// and work groups start in launch order.  Offsets are clamped to the tensors.
template <int R>
__device__ __forceinline__ bool seq_unit(const SeqArgs &a, int tile, SeqUnit &u) {
  int units, j;
  if (a.cu_q == nullptr) {
    u.nq = a.n_tokens / a.n_seqs;
    units = (u.nq * a.group + R - 1) / R;
    u.seq = tile / units;
    j = tile - u.seq * units;
    u.q0 = (int64_t)u.seq * u.nq;
    if (u.seq >= a.n_seqs) return false;
  } else {
    // every lane takes a sequence: a running count of units finds the one that holds `tile`
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    bool found = false;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
      const int s = s0 + lane;
      int first = 0, n = 0;
      if (s < a.n_seqs) {
        first = min(max(a.cu_q[s], 0), a.n_tokens);
        n = max(min(a.cu_q[s + 1], a.n_tokens) - first, 0);
      }
      const int mine = (n * a.group + R - 1) / R;
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
      }
      const uint64_t past = __ballot(before + upto > tile);
      if (past) {
        const int l = __ffsll((unsigned long long)past) - 1;
        u.seq = s0 + l;
        u.nq = __shfl(n, l);
        u.q0 = __shfl(first, l);
        units = __shfl(mine, l);
        j = (int)(tile - before) - (__shfl(upto, l) - units);
        found = true;
        break;
      }
      before += __shfl(upto, 63);
    }
    if (!found) return false;
  }
  u.seq = __builtin_amdgcn_readfirstlane(u.seq);
  u.nq = __builtin_amdgcn_readfirstlane(u.nq);
  u.q0 = __builtin_amdgcn_readfirstlane((int)u.q0);
  u.rows = u.nq * a.group;
  u.row0 = __builtin_amdgcn_readfirstlane((units - 1 - j) * R);
  if (a.kv_len) {
    u.nk = min(max(a.kv_len[u.seq], 0), a.capacity);
    u.k0 = 0;
  } else if (a.cu_k) {
    const int first = min(max(a.cu_k[u.seq], 0), a.n_keys);
    u.k0 = first;
    u.nk = max(min(a.cu_k[u.seq + 1], a.n_keys) - first, 0);
  } else {
    u.k0 = u.q0;
    u.nk = u.nq;
  }
  // (loads from memory that the kernel might write: uniform all the same)
  u.k0 = __builtin_amdgcn_readfirstlane((int)u.k0);
  u.nk = __builtin_amdgcn_readfirstlane(u.nk);
  return true;
}

// Keys that query i of the unit's sequence sees: the first of them up to this count.
__device__ __forceinline__ int seen_keys(const SeqArgs &a, const SeqUnit &u, int i) {
  if (a.block == 0) return u.nk;
  const int p = u.nk - u.nq + i;
  if (p < 0) return 0;
  // (below 2^32: p / block + 1 blocks end at most `block` behind p)
  const uint32_t end = ((uint32_t)p / (uint32_t)a.block + 1) * (uint32_t)a.block;
  return (int)min(end, (uint32_t)u.nk);
}

}  // namespace dev
}  // namespace hc
