// Gradients of the attention over packed sequences with a window: the kernels, which hc_window_grad64.hip and
// hc_window_grad128.hip compile for their head sizes, with matrix results in vector and in accumulation registers.
#pragma once

#include "hc_mask.h"
#include "hc_window.h"

namespace hc {
namespace {
using namespace dev;

// With P = exp(s q k^T - lse) and dS = P (dO V^T - rowsum(dO O)):
//   dV = P^T dO,  dK = s dS^T Q,  dQ = s dS K.
// Two kinds of units: one keeps keys and values of a run of keys and walks the queries that see them (dK, dV), the other keeps
// queries and their output gradients and walks their keys (dQ).  Both form the scores again, which is 7 products where
// 5 would do; in return nothing is added up through memory, and the order of every sum is fixed.
//
// Roundings.  P and dS are rounded to bf16, the operand type of their products (wider types run at a fraction of its rate); all
// sums are in 32 bits, and so is lse.  rowsum(dO O) is of the forward pass's output as it was rounded, so that dS of a row is off by one
// small offset.  Against 64 bits dQ and dK are off by 0.0024 to 0.0029 of their size (dS alone rounded: 0.0024; in 32 bits
// throughout, with the result rounded: 0.0017), most where a row sees few keys or weighs few of them.
//
// Both are one scheme.  A wave keeps two stationary operands B1, B2 (32 columns each, in registers as
// matrix operands) and walks tiles of two streamed tensors A1, A2 (64 rows, in LDS):
//   S = A1 B1 and T = A2 B2 (32 rows x 32 columns), then P and dS from them, and
//   C1 += A^T P or dS with a streamed tensor transposed: for that the LDS is read with the transposing
//   read, 16 lanes fetching 4 rows x 16 dims and each getting 4 rows of one dim.
// Rows are fed to S and T with bits 2 and 3 of their number swapped, so that a lane half g ends up with rows
// 8 g .. 8 g + 7 of every 16 (see hc_device.h), in the order that the second products contract.
//
// Bound by the matrix cores and the power that they draw with 128-dim heads: forward and gradients of a clip of three 480P blocks (14040
// tokens, 12 heads, a block sees itself and the first) 2.75 to 2.9 ms, by the card, the gradients 2.1-2.2 ms of it, 1.05-1.1 PFLOP/s of the 7 products, cores busy 53%
// at 2.0 GHz.  One wave on a SIMD, so that an operand and all sums stay in its 512 registers; two waves, with half of
// them, took 7% longer, and left no room for operands that are read 7 products ahead.  Without its copies a step would be 11%
// faster, without vector instructions 16%, without LDS reads 10% (timed apart).  64-dim heads: two waves on a SIMD; six prompts of
// 4000 tokens together (4 x 3 heads, window 512) 45 us, cores busy 26%: exponentials, masks and products of a wave in turn, and
// 1.5 waves on a SIMD at the mean.
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 64;        // streamed rows of a tile

// Position of 16-byte chunk c of row r of a streamed tile.  Both reads of it want different banks: 16 rows at one
// chunk (a score operand), and 4 neighbouring rows at 64 bytes (a transposing read).
template <int D>
__device__ __forceinline__ int tswz(int r, int c) {
  return c ^ (D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3));
}

// Streamed tiles in LDS: a ring of them, two tensors each.  Addresses are a lane's own part, and constants.
constexpr int kRing = 4;
// Operands of a step are read so many products ahead: each feeds one product of 32 cycles, and a read takes longer than
// four.  (64-dim heads run two waves on a SIMD, which fill in for each other.  The ring of operands comes around with every step.)
template <int D>
constexpr int kAhead = D == 128 ? 7 : 3;
template <int D>
struct Streamed {
  static constexpr int BYTES = kTile * D * 2, SLOT = 2 * BYTES;
  uint16_t x[kRing][2][kTile * D];
};
// (The numbers beside the rows are those of keys' units: the rows' logarithms, rowsum(dO O).)
template <int D>
struct Shared {
  __attribute__((aligned(1024))) Streamed<D> tiles;
  __attribute__((aligned(1024))) float rows[kRing][2][kTile];
};
using lds8 = const __attribute__((address_space(3))) bf16x8 *;
typedef short s16x4 __attribute__((ext_vector_type(4)));
using ldst = __attribute__((address_space(3))) s16x4 *;
using ldsf4 = const __attribute__((address_space(3))) f32x4 *;
// The products S and T.  128-dim heads: in inline assembly, with their stationary operand in the accumulation registers; as
// the compiler places it, that operand is copied for every product.  (tests/test_window_code.py looks at the distances between these
// products, what they read and what reads them.)  64-dim heads have vector registers for everything.
template <int D>
__device__ __forceinline__ void mfma_first(f32x16 &c, bf16x8 a, const bf16x8 &b) {
  if constexpr (D == 128) asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "a"(b));
  else c = mfma32(a, b, c);
}
template <int D>
__device__ __forceinline__ void mfma_first(f32x16 &c, bf16x8 a, const bf16x8 &b, const f32x16 &from) {
  // (a product reads what a vector instruction wrote 2 wait states before at the earliest: `from` may be a copy)
  if constexpr (D == 128) asm("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %3" : "=&v"(c) : "v"(a), "a"(b), "v"(from));
  else c = mfma32(a, b, from);
}
// Matrix results in their registers before vector instructions use them: a 32x32x16 product needs at most 18 wait states.  (The
// first wait is for copies that the compiler puts before an instruction that names the registers.)
template <int D>
__device__ __forceinline__ void settle(f32x16 &s, f32x16 &t) {
  if constexpr (D != 128) return;
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3");
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 3" : "+v"(s), "+v"(t));
}
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

template <int D>
struct Reader {
  uint32_t row, turn, turn4;           // of a lane, in bytes
  __device__ __forceinline__ explicit Reader(int lane) {
    const int n = lane & 31, g = lane >> 5, gl = lane >> 4, i = lane & 15;
    row = (uint32_t)(kperm(n) * D * 2 + tswz<D>(kperm(n), g) * 16);
    const int r = 8 * (gl / 2) + i / 4, chunk = 2 * (gl % 2) + (i % 4) / 2;
    turn = (uint32_t)(r * D * 2 + tswz<D>(r, chunk) * 16 + (i % 2) * 8);
    turn4 = (uint32_t)((r + 4) * D * 2 + tswz<D>(r + 4, chunk) * 16 + (i % 2) * 8);
  }
  // Operand i of a block's first products, whose tile is at `at` + row: dims 16 (i / 2) of its 32 rows, of tensor i % 2.
  static __device__ __forceinline__ bf16x8 first(uint32_t at, int i) {
    return *(lds8)(uintptr_t)((at ^ (uint32_t)(32 * (i / 2))) + (uint32_t)(i % 2 * Streamed<D>::BYTES));
  }
  // Operand of its second products, `at` and `at4` + turn and turn4: dims 32 db .. of rows 16 c .., transposed.
  static __device__ __forceinline__ bf16x8 second(uint32_t at, uint32_t at4, int tensor, int c, int db) {
    const uint32_t off = (uint32_t)(tensor * Streamed<D>::BYTES + c * 16 * D * 2), x = (uint32_t)(64 * db);
    struct { s16x4 a, b; } w;
    w.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)((at ^ x) + off));
    w.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)((at4 ^ x) + off));
    return __builtin_bit_cast(bf16x8, w);
  }
};

// Two DMA instructions (see hc_device.h) from base + a (bytes) and base + 1024 + b, behind a wait that covers a base which a
// vector instruction put into its scalar registers just before: 5 wait states, which the compiler does not count for
// inline assembly.
__device__ __forceinline__ void lds_dma16_two(const uint16_t *base, uint32_t a, uint32_t b, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %4\n\t"
      "s_nop 4\n\t"
      "global_load_lds_dwordx4 %1, %3\n\t"
      "global_load_lds_dwordx4 %2, %3 offset:0x400\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(a), "v"(b), "s"(base), "s"(lds)
      : "memory");
}

// 64 words to LDS by DMA, word i of the `left` behind p (the last repeats) to place i.
__device__ __forceinline__ void lds_dma4(const float *p, int left, int lane, uint32_t lds) {
  uint32_t saved;
  const uint32_t at = (uint32_t)min(lane, left - 1) * 4u;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %3\n\t"
      "s_nop 4\n\t"
      "global_load_lds_dword %1, %2\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(at), "s"(p), "s"(lds)
      : "memory");
}

// Copies tiles of one tensor to LDS by DMA: 64 rows of one head (those behind the last repeat it).  Instruction j of wave w
// moves 1 KB, the 8 or 4 rows from (N w + j) 512 / D on; a lane fetches the chunk that belongs at its 16 bytes.  (The base is
// 4 KB low, so that no offset goes below zero when 1024 j is taken off.)
template <int D>
struct Copier {
  static constexpr int RW = 512 / D, N = kTile / RW / kWaves;     // rows of an instruction, instructions of a wave
  static constexpr int PAIRS = N / 2;
  int lane, wave;
  uint32_t token;            // bytes from row to row: below 2^25, so that a row's offset stays below 2^31
  uint32_t at[N];            // of this lane, in a tile of `rows` rows
  int rows;
  __device__ __forceinline__ Copier(int64_t stride, int l, int w) : lane(l), wave(w), token((uint32_t)stride * 2u), rows(0) {
    of(kTile);
  }
  // For a tile with this many rows left.
  __device__ __forceinline__ void of(int left) {
    left = min(left, kTile);
    if (left == rows) return;
    rows = left;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int row = (N * wave + j) * RW + lane / (D / 8);
      at[j] = (uint32_t)min(row, left - 1) * token + (uint32_t)(tswz<D>(row, lane % (D / 8)) * 16 + 4096 - 1024 * j);
    }
  }
  // Instructions 2 i and 2 i + 1; p: the tile's first row.
  __device__ __forceinline__ void copy(const uint16_t *p, uint32_t tile, int i) const {
    lds_dma16_two(p - 2048 + i * 1024, at[2 * i], at[2 * i + 1], tile + (uint32_t)((wave * N + 2 * i) * 1024));
  }
  __device__ __forceinline__ void copy(const uint16_t *p, uint32_t tile) const {
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) copy(p, tile, i);
  }
};

// --- rowsum(dO O), and the logarithms in units of products of dims -------------------------------------------------
// A thread takes 8 dims of a row of a head; the 8 or 16 threads of a row add up.
template <int D>
__global__ __launch_bounds__(256) void grad_stats_kernel(GradArgs a) {
  constexpr int C = D / 8;
  const int heads = a.seq.kv_heads * a.seq.group;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i / C / heads;
  const int c = (int)(i % C), h = (int)(i / C % heads);
  const bool live = row < a.seq.n_tokens;
  float sum = 0.f;
  if (live) {
    const u32x4 x = gld16(a.dout + row * a.do_token + h * a.do_head + c * 8);
    const u32x4 y = gld16(a.seq.o + row * a.seq.o_token + h * a.seq.o_head + c * 8);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), sum);
      sum = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u), sum);
    }
  }
#pragma unroll
  for (int d = 1; d < C; d *= 2) sum += __shfl_xor(sum, d);
  if (live && c == 0) {
    const int64_t at = (int64_t)h * a.seq.n_tokens + row;
    // (where a product over dims begins from them, it ends as the logit less the logarithm, and as dP - rowsum)
    a.stats[at] = -a.lse[at] / a.scale;
    a.stats[(int64_t)heads * a.seq.n_tokens + at] = -sum;
  }
}

// P and dS of 8 rows as matrix operands
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const bf16x2 r = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, r);
}

// --- dK and dV: a work group takes 128 keys of a key head, each wave 32 --------------------------------
template <int D>
__device__ __forceinline__ void keys_unit(const GradArgs &a, int block, Shared<D> &lds) {
  constexpr int NKK = D / 16, NDB = D / 32;
  const SeqArgs &q = a.seq;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const int split = block % a.n_split;
  const int unit = block / a.n_split;
  const int tile = __builtin_amdgcn_readfirstlane(unit / q.kv_heads), head = unit - tile * q.kv_heads;
  SeqUnit u;
  if (!seq_unit<kGradKeys, true>(q, tile, u)) return;
  const int k0 = u.row0, k_last = min(k0 + kGradKeys, u.nk) - 1;
  const int key = k0 + 32 * wave + n;

  // The queries that see a key are a run of them: from its block's first on, and (but for the first tokens) before the block
  // whose window begins behind it.
  const int64_t off = (int64_t)u.nk - u.nq;          // position of query 0
  auto from = [&](int j) {
    return q.block ? (int)min(max((int64_t)((uint32_t)j / (uint32_t)q.block * (uint32_t)q.block) - off, (int64_t)0), (int64_t)u.nq) : 0;
  };
  auto until = [&](int j) {
    if (q.block == 0 || q.window == 0 || j < q.sinks) return u.nq;
    const uint32_t e = ((uint32_t)j + (uint32_t)q.window) / (uint32_t)q.block * (uint32_t)q.block;
    return (int)min(max((int64_t)e - off, (int64_t)0), (int64_t)u.nq);
  };
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int first = uniform(from(k0)), end = uniform(max(first, k0 < q.sinks ? u.nq : until(k_last)));
  const int nt = (end - first + kTile - 1) / kTile;    // tiles of every query head
  const int64_t items = (int64_t)nt * q.group;
  const int i0 = uniform((int)(items * split / a.n_split)), i1 = uniform((int)(items * (split + 1) / a.n_split));
  const int lo = from(min(key, u.nk - 1)), hi = until(min(key, u.nk - 1));

  bf16x8 kf[NKK], vf[NKK];
  {
    const int64_t row = u.k0 + min(key, u.nk - 1);
    const uint16_t *kp = q.k + row * q.k_token + head * q.k_head + 8 * g, *vp = q.v + row * q.v_token + head * q.v_head + 8 * g;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      kf[kk] = ld_g16(kp + 16 * kk);
      vf[kk] = ld_g16(vp + 16 * kk);
    }
  }
  f32x16 dk[NDB], dv[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dk[db] = dv[db] = f32x16{};

  Copier<D> copy_q(q.q_token, lane, wave), copy_o(a.do_token, lane, wave);
  using R = Reader<D>;
  const R reader(lane);
  const uint32_t tiles = lds_addr(&lds.tiles), rows = lds_addr(&lds.rows);
  auto slot = [&](int item) { return (uint32_t)((item - i0) % kRing); };
  // The tile that is copied next, moved on from tile to tile and head to head.  (Every wave copies one run of the rows' numbers, so
  // that all have as many copies in flight; two waves copy the same.)
  struct {
    const uint16_t *q, *o;
    const float *stats;
    int row;
  } next_tile;
  {
    const int h = head * q.group + i0 / max(nt, 1);
    next_tile.row = first + i0 % max(nt, 1) * kTile;
    const int64_t at = u.q0 + next_tile.row;
    next_tile.q = q.q + at * q.q_token + h * q.q_head;
    next_tile.o = a.dout + at * a.do_token + h * a.do_head;
    next_tile.stats = a.stats + (int64_t)(wave % 2 * q.kv_heads * q.group + h) * q.n_tokens + at;
  }
  // Copies of one tile, in 2 PAIRS + 1 parts.  There is one for every item, so that as many are always in flight: past the last
  // the last one is copied again, to a slot that nothing reads.
  auto prepare = [&] {
    copy_q.of(u.nq - next_tile.row);
    copy_o.of(u.nq - next_tile.row);
  };
  constexpr int PAIRS = Copier<D>::PAIRS;
  auto copy = [&](int item, int part) {
    const uint32_t to = tiles + slot(item) * Streamed<D>::SLOT;
    if (part < PAIRS) copy_q.copy(next_tile.q, to, part);
    else if (part < 2 * PAIRS) copy_o.copy(next_tile.o, to + Streamed<D>::BYTES, part - PAIRS);
    else lds_dma4(next_tile.stats, u.nq - next_tile.row, lane, rows + slot(item) * 512 + wave % 2 * 256);
  };
  auto move_on = [&](int item) {
    if (item + 1 >= i1) return;
    next_tile.row += kTile;
    next_tile.q += kTile * q.q_token;
    next_tile.o += kTile * a.do_token;
    next_tile.stats += kTile;
    if (next_tile.row >= end) {
      const int back = nt * kTile;
      next_tile.row = first;
      next_tile.q += q.q_head - back * q.q_token;
      next_tile.o += a.do_head - back * a.do_token;
      next_tile.stats += q.n_tokens - back;
    }
  };
  constexpr int COPIES = 2 * Copier<D>::N + 1;           // of a wave and tile

  // A step is block b of 32 rows: beside the products S and T of block b + 1 go the last exponentials of block b and what becomes
  // of them, beside its products dV and dK the first LATE exponentials of block b + 1, from the product on behind which S is there.
  // (All beside the first products they take longer than those: 16 of 16 cycles.)  Operands are read AHEAD products ahead.
  struct Scores {
    f32x16 s, t;
  };
  constexpr int NF = 2 * NKK, NS = 4 * NDB, EACH = 16 / NF;      // products of each half; elements of a first one
  constexpr int FROM = 3, PER = D == 128 ? 1 : 2, LATE = (NS - FROM) * PER;
  static_assert(LATE <= 16, "exponentials");
  constexpr int AHEAD = kAhead<D>, RO = AHEAD + 1;
  static_assert((NF + NS) % RO == 0, "the ring of operands");
  bf16x8 op[RO];
  const uint32_t lane_row = reader.row, turn = reader.turn, turn4 = reader.turn4;
  auto read_first = [&](uint32_t at, int i) { return R::first(at, i); };
  auto read_second = [&](uint32_t at, uint32_t at4, int j) {       // dV from the output gradients, dK from the queries
    return R::second(at, at4, 1 - j % 2, j / (2 * NDB), j / 2 % NDB);
  };
  // Where block qb of an item's tile is, and its rows' numbers.
  auto block_at = [&](int item, int qb) { return tiles + slot(item) * Streamed<D>::SLOT + (uint32_t)(qb * 32 * D * 2); };
  auto begin = [&](Scores &x, int item, int qb, int i) {         // rows 4 i .. of a lane's 16
    const uint32_t at = rows + slot(item) * 512 + (uint32_t)(qb * 128 + g * 32);
    const f32x4 l = *(ldsf4)(uintptr_t)(at + (uint32_t)(i / 2 * 64 + i % 2 * 16));
    const f32x4 d = *(ldsf4)(uintptr_t)(at + (uint32_t)(256 + i / 2 * 64 + i % 2 * 16));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x.s[4 * i + e] = l[e];
      x.t[4 * i + e] = d[e];
    }
  };
  // rows that do not see this lane's key get no weight, whether their exponential is there already or not
  auto mask = [&](Scores &x, int row) {
    const uint32_t from = (uint32_t)(row + 8 * g - lo), width = (uint32_t)(hi - lo);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (from + (uint32_t)(16 * (e / 8) + e % 8) >= width) x.s[e] = e < LATE ? 0.f : -INFINITY;
  };
  auto weight = [&](Scores &x, int e) { x.s[e] = __builtin_amdgcn_exp2f(x.s[e] * q.scale_log2); };
  auto step = [&](Scores &cur, Scores &nxt, int item, int qb) {
    const int item1 = item + qb;                         // of block b + 1
    const uint32_t next = block_at(item1, 1 - qb) + lane_row, after = block_at(item + 1, qb) + lane_row;
    const uint32_t here = block_at(item, qb) + turn, here4 = block_at(item, qb) + turn4;
    auto read_ahead = [&](int i) {
      const int r = i + AHEAD;
      op[r % RO] = r < NF ? read_first(next, r) : r < NF + NS ? read_second(here, here4, r - NF) : read_first(after, r - NF - NS);
    };
    u32x4 pf[2], df[2];
    float d0 = 0.f;
    // what is left of an element once its exponential is there
    auto rest = [&](int e) {
      const float d = cur.s[e] * cur.t[e];
      if (e % 2 == 0) {
        d0 = d;
      } else {
        pf[e / 8][e % 8 / 2] = pack2(cur.s[e - 1], cur.s[e]);
        df[e / 8][e % 8 / 2] = pack2(d0, d);
      }
    };
    fence();
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      read_ahead(i);
      mfma_first<D>(i % 2 == 0 ? nxt.s : nxt.t, op[i % RO], i % 2 == 0 ? kf[i / 2] : vf[i / 2]);
      fence();
#pragma unroll
      for (int e = EACH * i; e < EACH * (i + 1); ++e) {
        if (e >= LATE) weight(cur, e);
        if (e > 0) rest(e - 1);
      }
      fence();
    }
    rest(15);
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      read_ahead(NF + j);
      const int c = j / (2 * NDB), db = j / 2 % NDB;
      // (copies one by one: issued together they would wait for each other, and the products behind them)
      if (qb == 0 ? j < PAIRS : j <= PAIRS) copy(item + kRing - 1, qb * PAIRS + j);
      if (j % 2 == 0) dv[db] = mfma32(op[(NF + j) % RO], __builtin_bit_cast(bf16x8, pf[c]), dv[db]);
      else dk[db] = mfma32(op[(NF + j) % RO], __builtin_bit_cast(bf16x8, df[c]), dk[db]);
      if (j < 4) begin(cur, item + 1, qb, j);            // of block b + 2
      fence();
      if (j >= FROM) {
#pragma unroll
        for (int e = 0; e < PER; ++e) weight(nxt, (j - FROM) * PER + e);
        fence();
      }
    }
  };
  if (i0 < i1) {
    for (int i = i0; i < i0 + kRing - 1; ++i) {
      prepare();
#pragma unroll
      for (int part = 0; part <= 2 * PAIRS; ++part) copy(i, part);
      move_on(i);
    }
    // (the stationary operands, loaded before, are there only now)
    if constexpr (D == 128)
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+a"(kf[kk]), "+a"(vf[kk]));
    wait_vmcnt<2 * COPIES>();
    __syncthreads();
    Scores x, y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      begin(x, i0, 0, i);
      begin(y, i0, 1, i);
    }
#pragma unroll
    for (int i = 0; i < NF; ++i)
      mfma_first<D>(i % 2 == 0 ? x.s : x.t, read_first(block_at(i0, 0) + lane_row, i), i % 2 == 0 ? kf[i / 2] : vf[i / 2]);
    settle<D>(x.s, x.t);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) op[i] = read_first(block_at(i0, 1) + lane_row, i);
    int row = first + i0 % nt * kTile;                   // of the item
#pragma unroll
    for (int e = 0; e < LATE; ++e) weight(x, e);
    for (int item = i0; item < i1; ++item) {
      // tile item + 1 is there (tile item + 2 may be on its way), and every wave is done with tile item - 1
      wait_vmcnt<COPIES>();
      __syncthreads();
      prepare();
      const bool whole = __all(row >= lo && row + kTile <= hi);
      if (!whole) mask(x, row);
      step(x, y, item, 0);
      if (!whole) mask(y, row + 32);
      step(y, x, item, 1);
      row = row + kTile < end ? row + kTile : first;
      move_on(item + kRing - 1);
    }
    wait_vmcnt<0>();              // nothing is on its way to LDS that another work group may have next
  }

  // lane: key n of the wave, dims 32 db + 8 rq + 4 g .. + 3
  if (a.n_split > 1) {
    float *pp = a.part + ((int64_t)unit * a.n_split + split) * 2 * kGradKeys * D + (32 * wave + n) * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int dim = 32 * db + 8 * rq + 4 * g;
        *reinterpret_cast<f32x4 *>(pp + dim) = f32x4{dk[db][4 * rq], dk[db][4 * rq + 1], dk[db][4 * rq + 2], dk[db][4 * rq + 3]};
        *reinterpret_cast<f32x4 *>(pp + kGradKeys * D + dim) = f32x4{dv[db][4 * rq], dv[db][4 * rq + 1], dv[db][4 * rq + 2], dv[db][4 * rq + 3]};
      }
    return;
  }
  if (key >= u.nk) return;
  uint16_t *kp = a.dk + (u.k0 + key) * a.dk_token + head * a.dk_head, *vp = a.dv + (u.k0 + key) * a.dv_token + head * a.dv_head;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const int dim = 32 * db + 8 * rq + 4 * g;
      uint2 w;
      w.x = pack2(dk[db][4 * rq] * a.scale, dk[db][4 * rq + 1] * a.scale);
      w.y = pack2(dk[db][4 * rq + 2] * a.scale, dk[db][4 * rq + 3] * a.scale);
      *reinterpret_cast<uint2 *>(kp + dim) = w;
      w.x = pack2(dv[db][4 * rq], dv[db][4 * rq + 1]);
      w.y = pack2(dv[db][4 * rq + 2], dv[db][4 * rq + 3]);
      *reinterpret_cast<uint2 *>(vp + dim) = w;
    }
}

// Sums of the pieces of a key unit, in order: a thread takes 4 dims of a key.
template <int D>
__global__ __launch_bounds__(256) void grad_merge_kernel(GradArgs a) {
  constexpr int TR = D / 4, RW = 256 / TR, RP = kGradKeys / RW;
  const SeqArgs &q = a.seq;
  const int unit = blockIdx.x / RP;
  const int tile = __builtin_amdgcn_readfirstlane(unit / q.kv_heads), head = unit - tile * q.kv_heads;
  SeqUnit u;
  if (!seq_unit<kGradKeys, true>(q, tile, u)) return;
  const int lrow = (blockIdx.x % RP) * RW + threadIdx.x / TR, key = u.row0 + lrow;
  if (key >= u.nk) return;
  const int dim = threadIdx.x % TR * 4;
  const float *pp = a.part + (int64_t)unit * a.n_split * 2 * kGradKeys * D + lrow * D + dim;
  f32x4 dk = {0.f, 0.f, 0.f, 0.f}, dv = dk;
#pragma unroll 4
  for (int i = 0; i < a.n_split; ++i) {
    dk += *reinterpret_cast<const f32x4 *>(pp + (int64_t)i * 2 * kGradKeys * D);
    dv += *reinterpret_cast<const f32x4 *>(pp + ((int64_t)i * 2 + 1) * kGradKeys * D);
  }
  uint2 w;
  w.x = pack2(dk[0] * a.scale, dk[1] * a.scale);
  w.y = pack2(dk[2] * a.scale, dk[3] * a.scale);
  *reinterpret_cast<uint2 *>(a.dk + (u.k0 + key) * a.dk_token + head * a.dk_head + dim) = w;
  w.x = pack2(dv[0], dv[1]);
  w.y = pack2(dv[2], dv[3]);
  *reinterpret_cast<uint2 *>(a.dv + (u.k0 + key) * a.dv_token + head * a.dv_head + dim) = w;
}

// --- dQ: a work group takes 128 queries of a query head, each wave 32 ------------------------------------
template <int D>
__device__ __forceinline__ void queries_unit(const GradArgs &a, int block, Shared<D> &lds) {
  constexpr int NKK = D / 16, NDB = D / 32;
  SeqArgs q = a.seq;
  const int group = q.group;
  q.group = 1;                       // rows are the queries of one head
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const int heads = q.kv_heads * group;
  const int tile = __builtin_amdgcn_readfirstlane(block / heads), h = block - tile * heads, head = h / group;
  SeqUnit u;
  if (!seq_unit<kSeqRows>(q, tile, u)) return;
  const int row = u.row0 + 32 * wave + n, at = min(row, u.nq - 1);
  const Seen mine = seen_by(q, u, at);
  KeyTiles tiles(seen_by(q, u, u.row0), seen_by(q, u, min(u.row0 + kSeqRows, u.nq) - 1));
  tiles.first = __builtin_amdgcn_readfirstlane(tiles.first);
  tiles.gap = __builtin_amdgcn_readfirstlane(tiles.gap);
  tiles.lo_end = __builtin_amdgcn_readfirstlane(tiles.lo_end);
  tiles.hi_start = __builtin_amdgcn_readfirstlane(tiles.hi_start);
  bf16x8 qf[NKK], of[NKK];
  {
    const uint16_t *qp = q.q + (u.q0 + at) * q.q_token + h * q.q_head + 8 * g;
    const uint16_t *gp = a.dout + (u.q0 + at) * a.do_token + h * a.do_head + 8 * g;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      qf[kk] = ld_g16(qp + 16 * kk);
      of[kk] = ld_g16(gp + 16 * kk);
    }
  }
  // (see grad_stats_kernel: S and T begin from these)
  const float *sp = a.stats + (int64_t)h * q.n_tokens + u.q0 + at;
  const float lse = sp[0], delta = sp[(int64_t)q.n_tokens * heads];
  f32x16 from_s, from_t, dq[NDB];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    from_s[e] = lse;
    from_t[e] = delta;
  }
#pragma unroll
  for (int db = 0; db < NDB; ++db) dq[db] = f32x16{};

  Copier<D> copy_k(q.k_token, lane, wave), copy_v(q.v_token, lane, wave);
  using R = Reader<D>;
  const R reader(lane);
  const uint32_t lane_row = reader.row, turn = reader.turn, turn4 = reader.turn4;
  const uint16_t *kp = q.k + u.k0 * q.k_token + head * q.k_head, *vp = q.v + u.k0 * q.v_token + head * q.v_head;
  const uint32_t base = lds_addr(&lds.tiles);
  const int n_tiles = __builtin_amdgcn_readfirstlane(tiles.n);
  // (see keys_unit; past the last tile the last one again)
  constexpr int PAIRS = Copier<D>::PAIRS;
  const uint16_t *next_k, *next_v;
  auto prepare = [&](int t) {
    const int first = tiles.place(min(t, n_tiles - 1)) * kTile;
    next_k = kp + first * q.k_token;
    next_v = vp + first * q.v_token;
    copy_k.of(u.nk - first);
    copy_v.of(u.nk - first);
  };
  auto copy = [&](int t, int part) {
    const uint32_t to = base + (uint32_t)(t % kRing * Streamed<D>::SLOT);
    if (part < PAIRS) copy_k.copy(next_k, to, part);
    else copy_v.copy(next_v, to + Streamed<D>::BYTES, part - PAIRS);
  };
  constexpr int COPIES = 2 * Copier<D>::N;
  // A step as in keys_unit, with one second product for each operand: dQ.
  struct Scores {
    f32x16 s, t;
  };
  constexpr int NF = 2 * NKK, NS = 2 * NDB, EACH = 16 / NF;
  constexpr int FROM = 3, PER = 2, LATE = (NS - FROM) * PER;
  constexpr int AHEAD = kAhead<D>, RO = AHEAD + 1;
  static_assert((NF + NS) % RO == 0, "the ring of operands");
  bf16x8 op[RO];
  auto read_second = [&](uint32_t at, uint32_t at4, int j) { return R::second(at, at4, 0, j / NDB, j % NDB); };
  auto block_at = [&](int t, int kb) { return base + (uint32_t)(t % kRing * Streamed<D>::SLOT + kb * 32 * D * 2); };
  auto mask = [&](Scores &x, int key) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (!mine.sees(key + 8 * g + 16 * (e / 8) + e % 8)) x.s[e] = e < LATE ? 0.f : -INFINITY;
  };
  auto first_product = [&](Scores &x, int i, bf16x8 w) {
    const bf16x8 &b = i % 2 == 0 ? qf[i / 2] : of[i / 2];
    if (i < 2) mfma_first<D>(i % 2 == 0 ? x.s : x.t, w, b, i % 2 == 0 ? from_s : from_t);
    else mfma_first<D>(i % 2 == 0 ? x.s : x.t, w, b);
  };
  auto weight = [&](Scores &x, int e) { x.s[e] = __builtin_amdgcn_exp2f(x.s[e] * q.scale_log2); };
  auto step = [&](Scores &cur, Scores &nxt, int t, int kb) {
    const uint32_t next = block_at(t + kb, 1 - kb) + lane_row, after = block_at(t + 1, kb) + lane_row;
    const uint32_t here = block_at(t, kb) + turn, here4 = block_at(t, kb) + turn4;
    auto read_ahead = [&](int i) {
      const int r = i + AHEAD;
      op[r % RO] = r < NF ? R::first(next, r) : r < NF + NS ? read_second(here, here4, r - NF) : R::first(after, r - NF - NS);
    };
    u32x4 df[2];
    float d0 = 0.f;
    auto rest = [&](int e) {
      const float d = cur.s[e] * cur.t[e];
      if (e % 2 == 0) d0 = d;
      else df[e / 8][e % 8 / 2] = pack2(d0, d);
    };
    fence();
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      read_ahead(i);
      first_product(nxt, i, op[i % RO]);
      fence();
#pragma unroll
      for (int e = EACH * i; e < EACH * (i + 1); ++e) {
        if (e >= LATE) weight(cur, e);
        if (e > 0) rest(e - 1);
      }
      fence();
    }
    rest(15);
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      read_ahead(NF + j);
      if (j < PAIRS) copy(t + kRing - 1, kb * PAIRS + j);
      dq[j % NDB] = mfma32(op[(NF + j) % RO], __builtin_bit_cast(bf16x8, df[j / NDB]), dq[j % NDB]);
      fence();
      if (j >= FROM) {
#pragma unroll
        for (int e = 0; e < PER; ++e) weight(nxt, (j - FROM) * PER + e);
        fence();
      }
    }
  };
  if (n_tiles > 0) {
    for (int t = 0; t < kRing - 1; ++t) {
      prepare(t);
#pragma unroll
      for (int part = 0; part < 2 * PAIRS; ++part) copy(t, part);
    }
    if constexpr (D == 128)
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+a"(qf[kk]), "+a"(of[kk]));
    wait_vmcnt<2 * COPIES>();
    __syncthreads();
    Scores x, y;
#pragma unroll
    for (int i = 0; i < NF; ++i) first_product(x, i, R::first(block_at(0, 0) + lane_row, i));
    settle<D>(x.s, x.t);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) op[i] = R::first(block_at(0, 1) + lane_row, i);
#pragma unroll
    for (int e = 0; e < LATE; ++e) weight(x, e);
    for (int t = 0; t < n_tiles; ++t) {
      // tile t + 1 is there (tile t + 2 may be on its way), and every wave is done with tile t - 1
      wait_vmcnt<COPIES>();
      __syncthreads();
      prepare(t + kRing - 1);
      const int place = tiles.place(t);
      const bool whole = tiles.whole(place, q.sinks);
      if (!whole) mask(x, place * kTile);
      step(x, y, t, 0);
      if (!whole) mask(y, place * kTile + 32);
      step(y, x, t, 1);
    }
    wait_vmcnt<0>();
  }
  if (row >= u.nq) return;
  uint16_t *to = a.dq + (u.q0 + row) * a.dq_token + h * a.dq_head;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      uint2 w;
      w.x = pack2(dq[db][4 * rq] * a.scale, dq[db][4 * rq + 1] * a.scale);
      w.y = pack2(dq[db][4 * rq + 2] * a.scale, dq[db][4 * rq + 3] * a.scale);
      *reinterpret_cast<uint2 *>(to + 32 * db + 8 * rq + 4 * g) = w;
    }
}

// Both in one launch, units of keys first, which are the longer ones: neither needs the other, and the last of the ones run beside
// the first of the others.  (Forward and gradients, two launches and one: six prompts, window 512, 64 dims 104 and 81 us; two 480P
// blocks, 12 heads of 128 dims 1760 and 1630; 6000 tokens, 4 x 4 heads, causal 719 and 650; three 480P blocks, where power sets
// the pace, 2744 and 2728.)  Early keys and late queries, which have most to do under a causal mask, come first among their own
// (see seq_unit; queries from the first on: 650 -> 691, 2728 -> 2747).
template <int D>
__global__ __launch_bounds__(kThreads, D == 128 ? 1 : 2) void grad_kernel(GradArgs a) {
  __shared__ Shared<D> lds;
  const int keys = a.key_tiles * a.seq.kv_heads * a.n_split, block = (int)blockIdx.x;
  if (block < keys) keys_unit<D>(a, block, lds);
  else queries_unit<D>(a, block - keys, lds);
}

template <int D>
hipError_t launch(const GradArgs &a, hipStream_t s) {
  const int heads = a.seq.kv_heads * a.seq.group;
  const int64_t rows = (int64_t)a.seq.n_tokens * heads * (D / 8);
  if (rows > 0) hipLaunchKernelGGL(grad_stats_kernel<D>, dim3((uint32_t)((rows + 255) / 256)), dim3(256), 0, s, a);
  const int64_t blocks = (int64_t)a.key_tiles * a.seq.kv_heads * a.n_split + (int64_t)a.seq.tiles * heads;
  hipLaunchKernelGGL(grad_kernel<D>, dim3((uint32_t)blocks), dim3(kThreads), 0, s, a);
  if (a.n_split > 1 && a.key_tiles > 0)
    hipLaunchKernelGGL(grad_merge_kernel<D>, dim3((uint32_t)(a.key_tiles * a.seq.kv_heads * (kGradKeys * D / 1024))), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace hc
