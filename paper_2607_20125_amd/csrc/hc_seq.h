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

// Byte B of a word of scale codes as its power of two, for values2: the conversion takes the exponent
// field alone, so the neighbouring codes may stand in the other bits (tests/test_gpu_operator_values.py holds
// every scale beside others in each kernel; clearing them costs the 4-bit kernels 2%).
template <int B>
__device__ __forceinline__ float scale_of(uint32_t codes) {
  return __uint_as_float(B == 3 ? codes >> 1 : codes << (23 - 8 * B));
}

// The larger of two logits, NaN if one of them is: a row that sees a NaN has no other result, and
// the instruction for it takes three operands and needs no quieting of its inputs as fmaxf's does
// (34 instructions more for a tile of 64 keys in seq_attn_kernel).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// With the value 32 lanes away (the other half of a row's keys).
__device__ __forceinline__ float larger_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// One unit of work: rows row0 .. of a sequence (row r is query r / group).
struct SeqUnit {
  int seq;
  int row0, rows;          // first row, rows of the sequence
  int nq, nk;
  int64_t q0, k0;          // first query and key of the sequence in the packed tensors
};

// Queries and keys of sequence s, clamped to the tensors.
struct SeqSpan {
  int q0, nq, k0, nk;
};
__device__ __forceinline__ SeqSpan seq_span(const SeqArgs &a, int s) {
  SeqSpan p;
  if (a.cu_q) {
    p.q0 = min(max(a.cu_q[s], 0), a.n_tokens);
    p.nq = max(min(a.cu_q[s + 1], a.n_tokens) - p.q0, 0);
  } else {
    p.nq = a.n_tokens / a.n_seqs;
    p.q0 = s * p.nq;
  }
  if (a.kv_len) {
    p.k0 = 0;
    p.nk = min(max(a.kv_len[s], 0), a.capacity);
  } else if (a.cu_k) {
    p.k0 = min(max(a.cu_k[s], 0), a.n_keys);
    p.nk = max(min(a.cu_k[s + 1], a.n_keys) - p.k0, 0);
  } else {
    p.k0 = p.q0;
    p.nk = p.nq;
  }
  return p;
}

// Unit `tile` of the launch, in units of R rows; false if there is none.  Called by
// whole waves; results are uniform.  Work groups start in launch order, so what takes longest comes
// first: the later units of a sequence, which see the most keys under a causal mask, before the
// earlier ones, and up to 32 sequences by their keys.  (Ranking costs some 20 vector
// instructions a sequence and wave.  With units of 16 rows, whose waves share a SIMD by
// four, that was 5 us a work group for 48 sequences; there they stay in order.)
template <int R>
__device__ __forceinline__ bool seq_unit(const SeqArgs &a, int tile, SeqUnit &u) {
  SeqSpan p;
  int units, j;
  auto uniform = [](int x, int l) { return __builtin_amdgcn_readlane(x, l); };
  if (a.n_seqs == 1) {
    p = seq_span(a, 0);
    units = (p.nq * a.group + R - 1) / R;
    j = tile;
    u.seq = 0;
    if (j >= units) return false;
  } else if (R == kSeqRows && a.n_seqs <= 32) {
    // every lane takes a sequence and counts the units of those before it
    const int lane = threadIdx.x & 63;
    p = SeqSpan{0, 0, 0, 0};
    if (lane < a.n_seqs) p = seq_span(a, lane);
    const int mine = (p.nq * a.group + R - 1) / R;
    int64_t before = 0;
    for (int s = 0; s < a.n_seqs; ++s) {
      const int keys = uniform(p.nk, s), n = uniform(mine, s);
      if (keys > p.nk || (keys == p.nk && s < lane)) before += n;
    }
    const uint64_t here = __ballot(before <= tile && tile < before + mine);
    if (here == 0) return false;
    u.seq = __ffsll((unsigned long long)here) - 1;
    units = mine;
    j = (int)(tile - before);
  } else {
    // in their order: a running count of units finds the one that holds `tile`
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    bool found = false;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
      p = SeqSpan{0, 0, 0, 0};
      if (s0 + lane < a.n_seqs) p = seq_span(a, s0 + lane);
      const int mine = (p.nq * a.group + R - 1) / R;
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
      }
      const uint64_t past = __ballot(before + upto > tile);
      if (past) {
        u.seq = s0 + __ffsll((unsigned long long)past) - 1;
        units = mine;
        j = (int)(tile - before) - (upto - mine);
        found = true;
        break;
      }
      before += uniform(upto, 63);
    }
    if (!found) return false;
  }
  const int l = __builtin_amdgcn_readfirstlane(u.seq % 64);
  u.seq = __builtin_amdgcn_readfirstlane(u.seq);
  const int from = a.n_seqs == 1 ? 0 : l;
  u.nq = uniform(p.nq, from);
  u.q0 = uniform(p.q0, from);
  u.nk = uniform(p.nk, from);
  u.k0 = uniform(p.k0, from);
  u.rows = u.nq * a.group;
  u.row0 = (uniform(units, from) - 1 - uniform(j, from)) * R;
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

// What a work group has of the units: one of them, whole or a range of its keys.
struct SeqShare {
  int tile, head, split;
  bool cut;
  int64_t slot;            // of its partial result
  int32_t *place;          // where a cut unit's place is left for the merge
};
__device__ __forceinline__ SeqShare seq_share(const SeqArgs &a) {
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };    // (quotients come out of vector registers)
  SeqShare s;
  const int units = a.tiles * a.kv_heads, i = (int)blockIdx.x - a.whole;
  int unit = (int)blockIdx.x;
  s.split = 0;
  s.cut = i >= 0 && a.n_split > 1;
  if (i >= 0) {
    s.split = uniform(i / (units - a.whole));
    unit = a.whole + i - s.split * (units - a.whole);
  }
  s.tile = uniform(unit / a.kv_heads);
  s.head = unit - s.tile * a.kv_heads;
  s.slot = (int64_t)(unit - a.whole) * a.n_split + s.split;
  s.place = a.head + (int64_t)(unit - a.whole) * 4;
  return s;
}
// The range of key tiles that it takes: [t0, t1) of the nt that any row sees.  (Ranges of one length for
// every unit, more of them for longer sequences, give work groups that are alike but more
// that find nothing to do: 22.5 us instead of 18.9 for 48 sequences of 1 to 8192 cached tokens.)
__device__ __forceinline__ void key_range(const SeqArgs &a, const SeqUnit &u, const SeqShare &s, int nt, int &t0, int &t1) {
  t0 = 0;
  t1 = nt;
  if (!s.cut) return;
  t0 = (int)((int64_t)nt * s.split / a.n_split);
  t1 = (int)((int64_t)nt * (s.split + 1) / a.n_split);
  if (s.split == 0 && threadIdx.x == 0) {
    s.place[0] = (int)u.q0;
    s.place[1] = u.row0;
    s.place[2] = u.rows;
  }
}
// A unit that does not exist says so to the merge.
__device__ __forceinline__ void no_unit(const SeqShare &s) {
  if (s.cut && s.split == 0 && threadIdx.x == 0) s.place[2] = 0;
}
// Cut unit i in the merge.
__device__ __forceinline__ bool left_unit(const SeqArgs &a, int i, SeqUnit &u, int &head) {
  const int32_t *h = a.head + (int64_t)i * 4;
  u.q0 = h[0];
  u.row0 = h[1];
  u.rows = h[2];
  head = (a.whole + i) % a.kv_heads;
  return u.rows > 0;
}

// 32 finished rows of a wave on their way to memory: a lane of the matrix layout holds 4 dims of
// a row, which alone would be written 16 bytes of a row at a time; through LDS a row leaves
// in one piece.  Piece p of row r (8 bytes) is kept at p ^ 2 (r % 16).
template <int D>
struct OutRows {
  uint16_t *buf;                 // [32][D] of this wave's own
  __device__ __forceinline__ explicit OutRows(uint16_t *b) : buf(b) {}
  __device__ __forceinline__ void put(int r, int piece, float x0, float x1, float x2, float x3) {
    const bf16x2 x = {(__bf16)x0, (__bf16)x1}, y = {(__bf16)x2, (__bf16)x3};
    uint2 w;
    w.x = __builtin_bit_cast(uint32_t, x);
    w.y = __builtin_bit_cast(uint32_t, y);
    *reinterpret_cast<uint2 *>(buf + r * D + (piece ^ (2 * (r % (D / 8)))) * 4) = w;
  }
  // rows `first` .. first + 31 of the unit
  __device__ __forceinline__ void store(const SeqArgs &a, const SeqUnit &u, int head, int first, int lane) {
    constexpr int C = D / 8;     // 16-byte chunks of a row
#pragma unroll
    for (int i = 0; i < 32 * C / 64; ++i) {
      const int r = i * (64 / C) + lane / C, c = lane % C;
      const int row = u.row0 + first + r;
      const u32x4 w = *reinterpret_cast<const u32x4 *>(buf + r * D + (c ^ (r % C)) * 8);
      if (row < u.rows) {
        const int qi = row / a.group, qh = head * a.group + (row - qi * a.group);
        *reinterpret_cast<u32x4 *>(a.o + (u.q0 + qi) * a.o_token + qh * a.o_head + c * 8) = w;
      }
    }
  }
};

}  // namespace dev
}  // namespace hc
