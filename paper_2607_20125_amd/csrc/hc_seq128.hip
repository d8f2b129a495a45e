// Attention over sequences for 128-dim heads on waves of 64 rows: packed keys and values in bf16, or the 4-bit cache;
// with a window and first tokens, packed or in pages.
#include "hc_mask.h"
#include "hc_window.h"

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// One work group: 128 rows (queries times query heads of one key head) of a sequence on two
// waves of 64; two work groups share a CU (2 x 80 KB of LDS), one wave per SIMD.
//
// The arithmetic and its order are those of the dense kernel with 64 queries per wave
// (hc_dense128.hip): a step is 32 slots of two products each (16 of S(t+1) = K(t+1) Q^T, 16
// of O += V(t) P(t)), each with one pair of probabilities and one operand read three slots
// ahead, a fixed-offset softmax first and a running max where that does not stand; probabilities
// are rounded to bf16 for the products, and the row sums are of the rounded ones (see hc_seq.hip).  What
// differs:
//  * Rows are (query, head) pairs, each with its own count of keys, and the tiles that not every row
//    sees whole run masked, outside the written-out steps.
//  * V arrives token by token.  Its tile keeps that order in LDS, and the V^T operand is read with
//    the transposing read: 16 lanes fetch 4 tokens x 16 dims and each gets 4 tokens of
//    one dim.  Position p of row r holds 16-byte chunk p ^ 4 (r % 4), so that the 4
//    rows of such a read fall on different banks.
//  * Packed tiles are copied to LDS by DMA; 4-bit tiles go through registers, one
//    word (8 dims of a token, or 4 dims of two tokens) converted every second slot: V(t+1) beside
//    S(t+1), K(t+3) beside PV(t).
//
// Measured: a clip of four 480P blocks (18720 tokens, 12 heads, block-causal) 1.15 ms, 1.17 PFLOP/s, matrix cores
// busy 74% of cycles where power sets the clock; the waves of 32 rows (hc_seq.hip) took 1.59 ms.  A
// 480P block over its 4-bit window 0.83-0.90 ms, 1.05-1.14 PFLOP/s: conversions and their LDS
// writes take the issue slots that a step has left (58% busy), so a tile takes 27% more cycles than a packed one.
// Copies of the next tiles behind a branch instead of a rule for whole steps: 3.5% slower.
//
// With a window, or pages: written-out steps run over the whole tiles among the first tokens, and over those of the window;
// single steps, masked where they have to be, before, between and behind them.  (One nested loop over both kept more alive
// than the registers hold: 1.50 ms instead of 1.08.)  Pages: each copy is of a run of 16 rows, whose place comes by a scalar load a tile
// ahead.  A clip of four 480P blocks, window of two blocks and the first: 1.03 to 1.12 ms, by the card, 1.08 to 1.17 PFLOP/s, cores busy
// 66%; five prompts' 2500 rows over pages of 32, window 4096, 8 x 4 heads: 164-194 us, 0.8-0.9 PFLOP/s, cores busy 47%: masked steps at
// both ends of a window, and 968 work groups of uneven length on 512 places.  With logarithms, 64 additions more a tile: a clip
// of three blocks, window of one and the first, 635 us, cores busy 60%; without 596, 63%.
// ---------------------------------------------------------------------------
constexpr int kPre = 6;      // pairs of the next tile formed during PV
constexpr int kAhead = 3;    // operand reads in flight
constexpr int kCheckTile = 8;   // units of 4 kCheckTile tiles or more look at their row sums here

__device__ __forceinline__ void mfma_score(f32x16 &c, bf16x8 a, const bf16x8 &q, bool first) {
  if (first) asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(c) : "v"(a), "a"(q));
  else asm("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "a"(q));
}
__device__ __forceinline__ void fence() { __builtin_amdgcn_sched_barrier(0); }

// Four DMA instructions into consecutive 1 KB of LDS: instruction j moves 16 bytes per lane
// from base[j] + a[j] (bytes) + 1024 j to LDS lds + 1024 j + 16 lane (see hc_device.h).
// The wait covers a base that a vector instruction put into its scalar registers just
// before (a spilled one is brought back that way): 5 wait states, which the compiler
// does not count for inline assembly.
__device__ __forceinline__ void lds_dma16_offsets(const uint16_t *base, const uint32_t *a, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %6\n\t"
      "s_nop 4\n\t"
      "global_load_lds_dwordx4 %1, %5\n\t"
      "global_load_lds_dwordx4 %2, %5 offset:0x400\n\t"
      "global_load_lds_dwordx4 %3, %5 offset:0x800\n\t"
      "global_load_lds_dwordx4 %4, %5 offset:0xc00\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "s"(base), "s"(lds)
      : "memory");
}
__device__ __forceinline__ void lds_dma16_bases(const uint16_t *base, int64_t step, uint32_t a, uint32_t lds) {
  const uint16_t *b1 = base + step, *b2 = base + 2 * step, *b3 = base + 3 * step;
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %6\n\t"
      "s_nop 4\n\t"
      "global_load_lds_dwordx4 %1, %2\n\t"
      "global_load_lds_dwordx4 %1, %3 offset:0x400\n\t"
      "global_load_lds_dwordx4 %1, %4 offset:0x800\n\t"
      "global_load_lds_dwordx4 %1, %5 offset:0xc00\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(a), "s"(base), "s"(b1), "s"(b2), "s"(b3), "s"(lds)
      : "memory");
}

// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const uint16_t *uniform_ptr(const uint16_t *p) {
  const uint64_t x = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (const uint16_t *)((uint64_t)hi << 32 | lo);
}

// LOGS: the logarithms of the row sums too (see hc_seq.hip).
template <Keys SRC, bool LOGS = false>
__device__ __forceinline__ void attend128(const SeqArgs &a) {
  constexpr bool QUANT = SRC == Keys::kQuant, PAGED = SRC == Keys::kPaged, WINDOW = PAGED || SRC == Keys::kWindow;
  constexpr int D = 128, NQB = 2, KT = kSeqKeys, NKK = D / 16, NDB = D / 32;
  constexpr int TILE = KT * D;               // elements per tile
  constexpr int RK = 2, RV = 3;              // ring buffers
  static_assert(kSeqRows == 32 * 2 * NQB && KT == 64, "unit shape");
  __shared__ __attribute__((aligned(1024))) uint16_t sK[RK][TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sV[RV][TILE];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const SeqShare share = seq_share(a);
  const int head = share.head;
  SeqUnit u;
  if (!seq_unit<kSeqRows>(a, share.tile, u)) return no_unit(share);

  // this lane's rows wave 64 + 32 qb + n of the unit; a row behind the last repeats it
  int hi[NQB];               // keys it sees
  int start[NQB];            // with a window: those from here on and the first tokens
  bf16x8 qf[NQB][NKK];
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int at = min(u.row0 + wave * 64 + qb * 32 + n, u.rows - 1);
    const int qi = at / a.group, qh = head * a.group + (at - qi * a.group);
    if constexpr (WINDOW) {
      const Seen mine = seen_by(a, u, qi);
      hi[qb] = mine.end;
      start[qb] = mine.start;
    } else {
      hi[qb] = seen_keys(a, u, qi);
      start[qb] = 0;
    }
    const uint16_t *qp = a.q + (u.q0 + qi) * a.q_token + qh * a.q_head;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) qf[qb][kk] = ld_g16(qp + 16 * kk + 8 * g);
  }
  // Q in its registers before any DMA is issued (issued behind it, the copies of the first
  // tiles would be waited for with it: 3% slower where key ranges are short)
  wait_vmcnt<0>();
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+a"(qf[qb][kk]));
  const float sl2 = a.scale_log2;

  // The key range: nt tiles from tile t0 on.  Tiles below `plain` are seen whole by every row
  // (seen_keys grows with the query).
  const int last = min(u.row0 + kSeqRows, u.rows) - 1;
  auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  int lo_all = 0, nt_all;
  KeyTiles tiles(Seen{}, Seen{});
  if constexpr (WINDOW) {
    tiles = KeyTiles(seen_by(a, u, u.row0 / a.group), seen_by(a, u, last / a.group));
    tiles.first = uniform(tiles.first);
    tiles.gap = uniform(tiles.gap);
    tiles.lo_end = uniform(tiles.lo_end);
    tiles.hi_start = uniform(tiles.hi_start);
    tiles.lo_start = uniform(tiles.lo_start);
    tiles.hi_end = uniform(tiles.hi_end);
    tiles.hi_sink = uniform(tiles.hi_sink);
    nt_all = tiles.n;
  } else {
    lo_all = seen_keys(a, u, u.row0 / a.group);
    const int hi_all = seen_keys(a, u, last / a.group);
    nt_all = (hi_all + KT - 1) / KT;
  }
  int t0, t1;
  key_range(a, u, share, nt_all, t0, t1);
  t0 = __builtin_amdgcn_readfirstlane(t0);
  const int nt = __builtin_amdgcn_readfirstlane(t1 - t0);
  const int plain = __builtin_amdgcn_readfirstlane(lo_all / KT - t0);
  const int nk = u.nk - (WINDOW ? 0 : t0 * KT);      // keys of the sequence from tile t0 on; with a window, all
  // Place of the range's tile t: in the sequence with a window, else from tile t0 on; and whether every row sees it whole.
  auto place = [&](int t) { return WINDOW ? tiles.place(t0 + t) : t; };
  auto whole = [&](int t) {
    if constexpr (WINDOW) return tiles.whole(place(t), a.sinks);
    else return t < plain;
  };
  // With a window: the tile behind the run of whole tiles that t is in.
  auto whole_until = [&](int t) {
    const int p = place(t);
    const bool joined = tiles.hi_start <= a.sinks;       // (every key before the first row's end)
    const int until = joined || p * KT >= tiles.hi_start ? tiles.lo_end / KT - (p >= tiles.first ? tiles.gap : 0)
                                                         : min(a.sinks, tiles.lo_end) / KT;
    return until - t0;
  };

  // --- tiles: packed -----------------------------------------------------------------
  // Wave instruction j of a wave fills LDS rows 4 (8 wave + j) .. + 3, 16 chunks each.  K:
  // row r holds key (r & ~31) | kperm(r & 31), position p chunk kswz(r, p); instructions j and
  // j + 4 differ by 16 keys.  V: row r holds token r, position p chunk p ^ 4 (r % 4);
  // instructions differ by 4 tokens.  (The K base is 8 KB low, so that no offset goes
  // below zero when 1024 j is taken off.)
  const uint16_t *kbase = nullptr, *vbase = nullptr;
  uint32_t ka[4], va = 0;
  const uint32_t k_dst = lds_addr(&sK[0][wave * 8 * 512]);
  const uint32_t v_dst = lds_addr(&sV[0][wave * 8 * 512]);
  auto k_to = [&](int t) { return k_dst + (uint32_t)((t % RK) * TILE * 2); };
  auto v_to = [&](int t) { return v_dst + (uint32_t)((t % RV) * TILE * 2); };
  const int dma_row = lane >> 4, dma_pos = lane & 15;
  auto k_key = [&](int j) {                  // key of this lane in instruction j
    const int r = 4 * (8 * wave + j) + dma_row;
    return (r & ~31) | kperm(r & 31);
  };
  auto k_chunk = [&](int j) { return kswz<D>(4 * (8 * wave + j) + dma_row, dma_pos); };
  const int v_chunk = dma_pos ^ (4 * dma_row);
  const int wave_key = PAGED ? 0 : 32 * wave;       // (pages: rows count from their run of 16)
  if constexpr (!QUANT) {
    if constexpr (PAGED) {
      kbase = uniform_ptr(a.k + head * a.k_head);
      vbase = uniform_ptr(a.v + head * a.v_head);
    } else {
      const int64_t from = WINDOW ? 0 : (int64_t)t0 * KT;
      kbase = uniform_ptr(a.k + (u.k0 + from) * a.k_token + head * a.k_head);
      vbase = uniform_ptr(a.v + (u.k0 + from) * a.v_token + head * a.v_head);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      ka[j] = (uint32_t)(k_key(j) - 32 * wave + wave_key) * (uint32_t)a.k_token * 2u + (uint32_t)(k_chunk(j) * 16 + 8192 - 1024 * j);
    va = (uint32_t)(wave_key + dma_row) * (uint32_t)a.v_token * 2u + (uint32_t)(v_chunk * 16);
  }
  // Pages: where run 2 wave + half of tile t is, by a scalar load.  A run that has no page and that no row sees (its keys are
  // masked: pages that the window has passed) is read at a run in place of it whose 16 keys all were stored; one that
  // a row does see is noted.
  struct Run {
    int page, run;
  };
  bool gone = false;
  typedef const int32_t __attribute__((address_space(4))) *sptr;
  const sptr entries = PAGED ? (sptr)(uintptr_t)(a.table + (int64_t)u.seq * a.table_seq) : sptr();
  auto entry = [&](int run) { return entries[(run << 4) >> a.page_shift]; };
  auto present = [&](int p) { return (uint32_t)p < (uint32_t)a.n_pages; };
  Run stand_in{0, 0};
  if constexpr (PAGED) {
    if (nt > 0) {
      stand_in.run = max(tiles.hi_end / 16 - 1, 0);
      stand_in.page = entry(stand_in.run);
      if (!present(stand_in.page)) stand_in = Run{0, 0};
    }
  }
  auto run_in = [&](int t, int half) -> Run {
    if constexpr (!PAGED) return Run{0, 0};
    const int run = run_of(u, place(t), 2 * wave + half), p = entry(run);
    if (present(p)) return Run{p, run};
    const bool seen = run * 16 < tiles.hi_sink || (run * 16 + 16 > tiles.lo_start && run * 16 < tiles.hi_end);
    gone = gone || seen || stand_in.run == 0;
    return stand_in;
  };
  // its first row
  auto run_at = [&](const uint16_t *base, int64_t page_stride, int64_t token, Run r) {
    return base + r.page * page_stride + run_token(a, r.run) * token;
  };
  // (instruction 4 half + j; r: the run in pages)
  auto dma_k = [&](int t, int half, Run r) {
    const uint16_t *from;
    if constexpr (PAGED) from = run_at(kbase, a.k_page, a.k_token, r);
    else from = kbase + ((int64_t)place(t) * KT + 16 * half) * a.k_token;
    lds_dma16_offsets(from - 4096, ka, k_to(t) + 4096 * half);
  };
  auto dma_v = [&](int t, int half, Run r) {
    const uint16_t *from;
    if constexpr (PAGED) from = run_at(vbase, a.v_page, a.v_token, r);
    else from = vbase + ((int64_t)place(t) * KT + 16 * half) * a.v_token;
    lds_dma16_bases(from, 4 * a.v_token - 512, va, v_to(t) + 4096 * half);
  };

  // --- tiles: 4-bit ---------------------------------------------------------------------
  // A thread takes (token, 32 dims) items of K and (8 tokens, 4 dims) items of V, two each, 32
  // tokens apart.
  const uint8_t *cbase = nullptr;
  u32x4 kraw[2], vraw[2];
  uint32_t ksc[2], vsc[2][2];
  uint32_t kw_at[4] = {}, vw_at[4] = {};     // for word m % 4 of K, token % 4 of V
  if constexpr (QUANT) {
    cbase = a.cache + ((int64_t)u.seq * a.kv_heads + head) * a.cache_head + (int64_t)t0 * qtile_bytes(D);
    const int key = tid / 4, r = (key & ~31) | kperm(key & 31);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      kw_at[m] = (uint32_t)(uintptr_t)(lvoid)&sK[0][0] + (uint32_t)(r * 256 + kswz<D>(r, 4 * (tid % 4) + m) * 16);
      vw_at[m] = (uint32_t)(uintptr_t)(lvoid)&sV[0][0] + (uint32_t)((tid / 32) * 8 * 256 + ((((tid % 32) ^ (tid / 32 % 2 * 16)) * 8) ^ (64 * m)));
    }
  }
  // (the second half of a wave takes the dims in the other order of halves: its rows are 8 further, on the
  // same banks)
  const int vd4 = (tid % 32) ^ (tid / 32 % 2 * 16);
  auto load_k = [&](int t) {
    const uint8_t *tp = cbase + (int64_t)t * qtile_bytes(D);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      kraw[e] = *(gptr16)(tp + (tid + 128 * e) * 16);
      ksc[e] = tp[qtile_k_scales(D) + tid + 128 * e];
    }
  };
  auto load_v = [&](int t) {
    const uint8_t *tp = cbase + (int64_t)t * qtile_bytes(D) + qtile_v(D);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      vraw[e] = *(gptr16)(tp + ((tid / 32 + 4 * e) * 32 + vd4) * 16);
      const uint2 s = *(const uint2 *)(tp + KT * D / 2 + (((tid / 32) + 4 * e) * 4 + vd4 / 8) * 8);
      vsc[e][0] = s.x;
      vsc[e][1] = s.y;
    }
  };
  // slots behind the sequence's end hold anything: their scale becomes the smallest, so that
  // a probability of 0 times their value is 0
  auto cut_v = [&](int t) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int left = nk - t * KT - 8 * (tid / 32 + 4 * e);
      if (left < 8) {
        vsc[e][0] = left >= 4 ? vsc[e][0] : left <= 0 ? 0u : vsc[e][0] & ((1u << (8 * left)) - 1u);
        vsc[e][1] = left <= 4 ? 0u : vsc[e][1] & ((1u << (8 * (left - 4))) - 1u);
      }
    }
  };
  using lds16w = __attribute__((address_space(3))) u32x4 *;
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  using lds8w = __attribute__((address_space(3))) u32x2 *;
  // word i of 8: item i / 4, its word i % 4
  auto put_k = [&](uint32_t slot, int i) {
    const int e = i / 4, m = i % 4;
    const uint32_t w = kraw[e][m];
    const float scale = __uint_as_float(ksc[e] << 23);
    *(lds16w)(uintptr_t)(kw_at[m] + slot + (uint32_t)(e * 32 * 256)) =
        u32x4{values2<0>(w, scale), values2<1>(w, scale), values2<2>(w, scale), values2<3>(w, scale)};
  };
  auto put_v = [&](uint32_t slot, int i) {
    const int e = i / 4, m = i % 4;              // tokens 2 m and 2 m + 1 of the item
    const uint32_t w = vraw[e][m], s = vsc[e][m / 2];
    const float sx = m % 2 ? scale_of<2>(s) : scale_of<0>(s), sy = m % 2 ? scale_of<3>(s) : scale_of<1>(s);
    const uint32_t at = slot + (uint32_t)((e * 32 + 2 * m) * 256);
    *(lds8w)(uintptr_t)(vw_at[2 * m % 4] + at) = u32x2{values2<0>(w, sx), values2<1>(w, sx)};
    *(lds8w)(uintptr_t)(vw_at[2 * m % 4 + 1] + at + 256) =
        u32x2{values2<2>(w, sy), values2<3>(w, sy)};
  };
  auto k_slot = [&](int t) { return (uint32_t)((t % RK) * TILE * 2); };
  auto v_slot = [&](int t) { return (uint32_t)((t % RV) * TILE * 2); };

  // One tile into its slot, any of them: by DMA (rows behind the end repeat the last one), or
  // loaded, converted and written here.
  auto fetch_k = [&](int t) {
    if constexpr (QUANT) {
      load_k(t);
#pragma unroll
      for (int i = 0; i < 8; ++i) put_k(k_slot(t), i);
    } else if ((place(t) + 1) * KT <= nk) {
      dma_k(t, 0, run_in(t, 0));
      dma_k(t, 1, run_in(t, 1));
    } else if constexpr (PAGED) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int run = run_of(u, place(t), 2 * wave + half) * 16 - place(t) * KT;      // its first key, of the tile
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          b[j] = (uint32_t)(min(k_key(4 * half + j), nk - 1 - place(t) * KT) - run) * (uint32_t)a.k_token * 2u +
                 (uint32_t)(k_chunk(4 * half + j) * 16 + 8192 - 1024 * j);
        lds_dma16_offsets(run_at(kbase, a.k_page, a.k_token, run_in(t, half)) - 4096, b, k_to(t) + 4096 * half);
      }
    } else {
      uint32_t b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        b[j] = (uint32_t)min(k_key(j), nk - 1 - place(t) * KT) * (uint32_t)a.k_token * 2u +
               (uint32_t)(k_chunk(j) * 16 + 8192 - 1024 * j);
      const uint16_t *from = kbase + (int64_t)place(t) * KT * a.k_token - 4096;
      lds_dma16_offsets(from, b, k_to(t));
      lds_dma16_offsets(from + 2048, b + 4, k_to(t) + 4096);
    }
  };
  auto fetch_v = [&](int t) {
    if constexpr (QUANT) {
      load_v(t);
      cut_v(t);
#pragma unroll
      for (int i = 0; i < 8; ++i) put_v(v_slot(t), i);
    } else if ((place(t) + 1) * KT <= nk) {
      dma_v(t, 0, run_in(t, 0));
      dma_v(t, 1, run_in(t, 1));
    } else if constexpr (PAGED) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int run = run_of(u, place(t), 2 * wave + half) * 16 - place(t) * KT;
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          b[j] = (uint32_t)(min(4 * (8 * wave + 4 * half + j) + dma_row, nk - 1 - place(t) * KT) - run) * (uint32_t)a.v_token * 2u +
                 (uint32_t)(v_chunk * 16 + 8192 - 1024 * j);
        lds_dma16_offsets(run_at(vbase, a.v_page, a.v_token, run_in(t, half)) - 4096, b, v_to(t) + 4096 * half);
      }
    } else {
      uint32_t b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        b[j] = (uint32_t)min(4 * (8 * wave + j) + dma_row, nk - 1 - place(t) * KT) * (uint32_t)a.v_token * 2u +
               (uint32_t)(v_chunk * 16 + 8192 - 1024 * j);
      const uint16_t *from = vbase + (int64_t)place(t) * KT * a.v_token - 4096;
      lds_dma16_offsets(from, b, v_to(t));
      lds_dma16_offsets(from + 2048, b + 4, v_to(t) + 4096);
    }
  };
  // what this wave has in flight has arrived, and then what every wave had
  auto arrived = [&] {
    wait_vmcnt<0>();
    __syncthreads();
  };

  f32x16 acc[NQB][NDB];
  float m_run[NQB], l_run[NQB];
  // Row sums of the fixed-offset pass on the matrix cores: a 16x16x32 product of a 0/1
  // selector with the P operand (see hc_dense128.hip).  Lane n < 16 then holds the sum
  // of row n in lacc[.][0], of n + 16 in lacc[.][1].
  f32x4 lacc[NQB];
  bf16x8 sel;
  {
    const int i = lane & 15, kg = lane >> 4;
    const float v = (i == 0 && (kg & 1) == 0) || (i == 1 && (kg & 1) == 1) ? 1.f : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sel[e] = (__bf16)v;
  }

  using Scores = f32x16[2][NQB];   // [32-key block][row block]
  using Probs = u32x4[4][NQB];     // [16-key chunk][row block]: 8 probabilities in bf16
  using lds8 = const __attribute__((address_space(3))) bf16x8 *;
  uint32_t k_at[NKK];
#pragma unroll
  for (int kk = 0; kk < NKK; ++kk)
    k_at[kk] = (uint32_t)(uintptr_t)(lvoid)&sK[0][n * D] +
               ((uint32_t)(kswz<D>(n, g) * 16) ^ (uint32_t)(32 * kk));
  auto ldk = [&](uint32_t slot, int i) -> bf16x8 {   // read i: 16 dims i / 2, key block i % 2
    return *(lds8)(uintptr_t)(k_at[i / 2] + slot + (uint32_t)(64 * D * (i % 2)));
  };
  // V operand: lane (group gl = lane / 16, i = lane % 16) fetches dims 16 (gl % 2) + 4 (i % 4) .. + 3
  // of token 8 (gl / 2) + i / 4 and, in a second read, of the token 4 further
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  using ldst = __attribute__((address_space(3))) s16x4 *;
  const int gl = lane >> 4, li = lane & 15;
  const uint32_t v_lane = (uint32_t)(uintptr_t)(lvoid)&sV[0][0] +
                          (uint32_t)((8 * (gl / 2) + li / 4) * 256 + (li / 4) * 64 + (gl % 2) * 32 + (li % 4) * 8);
  auto ldv = [&](uint32_t slot, int i) -> bf16x8 {   // read i: key chunk i / 4, 32 dims i % 4
    const uint32_t at = (v_lane ^ (uint32_t)((i % 4) * 64)) + slot;
    struct { s16x4 a, b; } r;
    r.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)(at + (uint32_t)((i / 4) * 16 * 256)));
    r.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)(at + (uint32_t)((i / 4) * 16 * 256 + 4 * 256)));
    return __builtin_bit_cast(bf16x8, r);
  };
  // matrix results in their registers before vector instructions use them: a
  // 32x32x16 product needs at most 18 wait states (the first wait is for copies that
  // the compiler puts before an instruction that names the registers)
  auto settle = [&](Scores &s) {
    fence();
    asm volatile("s_nop 15\n\ts_nop 3");
    fence();
    asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s[0][0]), "+v"(s[0][1]), "+v"(s[1][0]), "+v"(s[1][1]));
  };
  auto qk = [&](int t, Scores &s) {
#pragma unroll
    for (int i = 0; i < 2 * NKK; ++i) {
      const bf16x8 kf = ldk(k_slot(t), i);
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) mfma_score(s[i % 2][qb], kf, qf[qb][i / 2], i < 2);
    }
    settle(s);
  };
  // keys that a row does not see get no weight
  auto mask = [&](Scores &s, int t) {
    const int first = (WINDOW ? place(t) : t0 + t) * KT;
    if (!WINDOW || first + KT > tiles.lo_end) {
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        const int rem = hi[qb] - first - 8 * g;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)       // (kperm(8 (r / 4) + 4 g + r % 4) = 8 g + kperm(...) at g = 0)
          {
            if (32 * kb + kperm(8 * (r >> 2) + (r & 3)) >= rem) s[kb][qb][r] = -INFINITY;
            if (WINDOW && r % 8 == 7) fence();
          }
      }
    }
    if constexpr (WINDOW) {
      // those between the first tokens and the row's window
      if (first + KT > a.sinks && first < tiles.hi_start) {
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) {
          int low = first + 8 * g - a.sinks;
          uint32_t width = (uint32_t)max(start[qb] - a.sinks, 0);
          asm volatile("" : "+v"(low), "+v"(width));     // (or 32 differences stay in registers for the other rows)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
            {
              if ((uint32_t)(low + 32 * kb + kperm(8 * (r >> 2) + (r & 3))) < width) s[kb][qb][r] = -INFINITY;
              if (r % 8 == 7) fence();
            }
        }
      }
    }
  };
  // pair p of a tile's probabilities: key chunk p / 8, row block (p / 4) % 2,
  // elements 2 (p % 4) and the next
  auto score = [](const Scores &s, int p, int e) {
    return s[p / 16][(p / 4) % 2][8 * ((p / 8) % 2) + 2 * (p % 4) + e];
  };
  float e_run[NQB] = {};          // LOGS: this lane's half of its rows' sums
  auto pack = [&](Probs &pf, int p, float x0, float x1) {
    uint32_t r;
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(r) : "v"(x0), "v"(x1));
    pf[p / 8][(p / 4) % 2][p % 4] = r;
    if constexpr (LOGS) e_run[(p / 4) % 2] += x0 + x1;
  };
  auto probs = [](const Probs &pf, int chunk, int qb) { return __builtin_bit_cast(bf16x8, pf[chunk][qb]); };
  auto row_sums = [&](const Probs &pf, int chunk) {
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
      lacc[qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sel, probs(pf, chunk, qb), lacc[qb], 0, 0, 0);
  };

  // --- fixed-offset pass: each probability is 2^x for the logit x in log2 units,
  // with no row max, no subtraction and no rescale.  That is exact softmax
  // arithmetic as long as nothing overflows or underflows (checked below).
  float px0, px1;                 // the last pair, not yet packed
  bf16x8 kf[kAhead + 1];
  auto prob = [&](const Scores &s, int p, int e) {
    return __builtin_amdgcn_exp2f(score(s, p, e) * sl2);
  };
  // S(t+1), then PV(t), with the probabilities of tile t from pair kPre on and the
  // first kPre pairs of tile t+1 beside the products.  STEADY: tile t+4 exists, tile t+1 is
  // seen whole, kslot is a constant, and kf holds the first reads of K(t+1).
  auto step = [&](auto steady, int t, uint32_t kslot, Scores &cur, Scores &nxt, Probs &pf) {
    constexpr bool STEADY = decltype(steady)::value;
    const uint32_t vb = v_slot(t), vn = v_slot(t + 1);
    if constexpr (!STEADY) {
      if constexpr (QUANT) {
        cut_v(t + 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) put_v(vn, i);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) kf[i] = ldk(kslot, i);
    }
    fence();
    auto slot = [&](int i, auto &&product) {
      const int p = kPre + i;
      product(0);
      fence();
      const float y0 = p < 32 ? prob(cur, p, 0) : prob(nxt, p - 32, 0);
      const float y1 = p < 32 ? prob(cur, p, 1) : prob(nxt, p - 32, 1);
      fence();
      product(1);
      fence();
      pack(pf, (p - 1) % 32, px0, px1);
      px0 = y0;
      px1 = y1;
      fence();
    };
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + kAhead < 16) kf[(i + kAhead) % 4] = ldk(kslot, i + kAhead);
      else kf[(i + kAhead) % 4] = ldv(vb, i + kAhead - 16);
      if constexpr (STEADY && QUANT)
        if (i % 2 == 1) put_v(vn, i / 2);
      slot(i, [&](int qb) { mfma_score(nxt[i % 2][qb], kf[i % 4], qf[qb][i / 2], i < 2); });
    }
    // (scalar loads come back in any order, so every wait behind one is for all of the LDS reads too: here all are over anyway)
    Run kr[2] = {}, vr[2] = {};
    if constexpr (STEADY && PAGED) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        kr[i] = run_in(t + 3, i);
        vr[i] = run_in(t + 2, i);
      }
    }
    if constexpr (!QUANT) wait_vmcnt<0>();     // K(t+2) and V(t+1) landed
    __syncthreads();              // ... for every wave; S(t+1) and PV(t-1) are over
    if constexpr (!STEADY) {
      settle(nxt);
      if (!whole(t + 1)) mask(nxt, t + 1);
      if constexpr (QUANT) {
        // (K(t+3) is in its registers if it exists)
        if (t + 3 < nt) {
#pragma unroll
          for (int i = 0; i < 8; ++i) put_k(kslot, i);
        }
        if (t + 4 < nt) load_k(t + 4);
        if (t + 2 < nt) load_v(t + 2);
      } else {
        if (t + 3 < nt) fetch_k(t + 3);
        if (t + 2 < nt) fetch_v(t + 2);
      }
    } else if constexpr (QUANT) {
      load_v(t + 2);
    }
    fence();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i + kAhead < 16) kf[(i + kAhead) % 4] = ldv(vb, i + kAhead);
      else if constexpr (STEADY) kf[(i + kAhead) % 4] = ldk(kslot ^ (uint32_t)(TILE * 2), i + kAhead - 16);
      if constexpr (STEADY && QUANT) {
        if (i % 2 == 1) put_k(kslot, i / 2);
      } else if constexpr (STEADY) {
        if (i < 2) dma_k(t + 3, i, kr[i]);
        else if (i < 4) dma_v(t + 2, i - 2, vr[i - 2]);
      }
      slot(16 + i, [&](int qb) { acc[qb][i % 4] = mfma32(kf[i % 4], probs(pf, i / 4, qb), acc[qb][i % 4]); });
      if (i % 4 == 3) {
        row_sums(pf, i / 4);
        fence();
      }
    }
    if constexpr (STEADY && QUANT) load_k(t + 4);
  };
  // Whether a row sum is out of range already (NaN included).
  auto sums_over = [&](int t) -> bool {
    bool over = false;
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb)
      over = over || max(__float_as_uint(lacc[qb][0]), __float_as_uint(lacc[qb][1])) >
                         __builtin_bit_cast(uint32_t, 0x1p96f);
    over = __any(lane < 16 && over);
    // the waves agree through the V slot of tile t - 1: read by both, and
    // refilled only after the next step's barrier
    int *flag = reinterpret_cast<int *>(&sV[(t - 1) % RV][0]);
    __syncthreads();
    if (lane == 0) flag[wave] = over ? 1 : 0;
    __syncthreads();
    return (flag[0] | flag[1]) != 0;
  };
  // Returns false as soon as it cannot stand any more: row sums only grow, so one
  // above the bound after kCheckTile tiles (NaN included) stays above it, and the
  // rest of the pass would be for nothing.
  auto run_fixed = [&]() -> bool {
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) lacc[qb] = f32x4{};
    fetch_k(0);
    if (nt > 1) fetch_k(1);
    fetch_v(0);
    arrived();
    Scores sa, sb;
    Probs pf;
    qk(0, sa);
    if (!whole(0)) mask(sa, 0);
    __syncthreads();              // S(0) is over for every wave
    if (nt > 2) fetch_k(2);
    if constexpr (QUANT) {
      if (nt > 3) load_k(3);
      if (nt > 1) load_v(1);
    } else {
      if (nt > 1) fetch_v(1);
    }
    // a pair with its pack (an exp2 result needs one wait state before the pack)
    auto pair = [&](int p) {
      px0 = prob(sa, p, 0);
      px1 = prob(sa, p, 1);
      asm volatile("s_nop 1" : "+v"(px0), "+v"(px1));
    };
#pragma unroll
    for (int p = 0; p < kPre; ++p) {
      if (p) pack(pf, p - 1, px0, px1);
      pair(p);
    }
    int t = 0;
    if constexpr (WINDOW) {
      // Written-out steps, two at a time from an even tile on, for the whole tiles among the first tokens, then for those
      // of the window (which may be one run); single ones, masked where they have to be, before, between and behind.
      bool checked = nt < 4 * kCheckTile;
      auto steady = [&](int n_steady) -> bool {
        if (t + 1 >= n_steady) return true;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) kf[i] = ldk(TILE * 2, i);
        for (;;) {
          int stop = n_steady;
          if (!checked) stop = min(stop, max(t + 2, kCheckTile));
          for (; t + 1 < stop; t += 2) {
            step(std::true_type{}, t, TILE * 2, sa, sb, pf);
            step(std::true_type{}, t + 1, 0, sb, sa, pf);
          }
          if (t + 1 >= n_steady) return true;
          if (!checked && t >= kCheckTile) {
            checked = true;
            if (sums_over(t)) return false;
          }
        }
      };
      auto single = [&] {
        step(std::false_type{}, t, k_slot(t + 1), sa, sb, pf);
        ++t;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb) sa[kb][qb] = sb[kb][qb];
      };
      if (!steady(whole(1) ? min(nt - 4, whole_until(1) - 1) : 0)) return false;
      const int window = max((tiles.hi_start + KT - 1) / KT - tiles.gap - t0, 0);       // its first whole tile
      const int n_window = min(nt - 4, tiles.lo_end / KT - tiles.gap - t0 - 1);
      if (window > 0 && window < n_window) {
        while (t % 2 != 0 || t + 1 < window) single();
        if (!steady(n_window)) return false;
      }
      while (t + 1 < nt) single();
    } else {
      // the written-out steps end before the last four tiles and before the first masked one
      const int n_steady = min(nt - 4, plain - 1);
      if (t < n_steady - 1) {
        // (QUANT: K(2) was written without a barrier behind it, which the step's own one gives)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) kf[i] = ldk(TILE * 2, i);
        for (int stop = nt >= 4 * kCheckTile && n_steady > kCheckTile ? kCheckTile : n_steady;; stop = n_steady) {
          for (; t + 1 < n_steady && t < stop; t += 2) {   // two steps, so that the score sets swap roles
            step(std::true_type{}, t, TILE * 2, sa, sb, pf);
            step(std::true_type{}, t + 1, 0, sb, sa, pf);
          }
          if (stop == n_steady) break;
          if (sums_over(t)) return false;
        }
      }
      while (t + 1 < nt) {
        step(std::false_type{}, t, k_slot(t + 1), sa, sb, pf);
        ++t;
        if (t + 1 < nt) {
          step(std::false_type{}, t, k_slot(t + 1), sb, sa, pf);
          ++t;
        } else {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int qb = 0; qb < NQB; ++qb) sa[kb][qb] = sb[kb][qb];
        }
      }
    }
    // last tile: the rest of its probabilities, PV(nt - 1)
#pragma unroll
    for (int p = kPre; p < 32; ++p) {
      pack(pf, p - 1, px0, px1);
      pair(p);
    }
    pack(pf, 31, px0, px1);
    fence();
    asm volatile("s_nop 1");      // the last pack before the products
    fence();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const bf16x8 vf = ldv(v_slot(t), i);
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) acc[qb][i % 4] = mfma32(vf, probs(pf, i / 4, qb), acc[qb][i % 4]);
      if (i % 4 == 3) row_sums(pf, i / 4);
    }
    return true;
  };

  // --- running-max pass: the online softmax with lazy rescaling, tile by tile, for
  // the units whose fixed-offset pass does not stand
  auto run_max = [&] {
    const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int qb = 0; qb < NQB; ++qb) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) acc[qb][db] = f32x16{};
      m_run[qb] = kMInit;
      l_run[qb] = 0.f;
      e_run[qb] = 0.f;
    }
    __syncthreads();              // every wave is done with the slots
    // (an absent run's rows are copied from page 0 and do not count)
    fetch_k(0);
    fetch_v(0);
    for (int t = 0; t < nt; ++t) {
      arrived();                  // tile t is there, and tile t - 1 is over
      uint32_t hidden = 0;        // runs
      if constexpr (PAGED) hidden = absent_runs(a, page_entry(a, u, place(t), lane));
      if (t + 1 < nt) {
        fetch_k(t + 1);
        fetch_v(t + 1);
      }
      if constexpr (PAGED) {
        if (hidden) {             // a probability of 0 times 0 is 0
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (hidden >> (i / 2) & 1)
              *reinterpret_cast<u32x4 *>(&sV[t % RV][i * 1024 + tid * 8]) = u32x4{0, 0, 0, 0};
          __syncthreads();
        }
      }
      Scores s;
      Probs pf;
      qk(t, s);
      if (!whole(t)) mask(s, t);
      if constexpr (PAGED) {
        if (hidden)
#pragma unroll
          for (int qb = 0; qb < NQB; ++qb)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if (hidden >> (2 * kb + (r >> 3)) & 1) s[kb][qb][r] = -INFINITY;
      }
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        float m = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) m = larger(m, larger(s[0][qb][r], s[1][qb][r]));
        m = larger_xor32(m) * sl2;
        if (__any(m > m_run[qb] + kRescale)) {
          const float m_new = larger(m_run[qb], m);
          const float alpha = __builtin_amdgcn_exp2f(m_run[qb] - m_new);
          m_run[qb] = m_new;
          l_run[qb] *= alpha;
          e_run[qb] *= alpha;
#pragma unroll
          for (int db = 0; db < NDB; ++db) acc[qb][db] *= alpha;
        }
      }
#pragma unroll
      for (int p = 0; p < 32; ++p) {
        const int qb = (p / 4) % 2;
        const float x0 = __builtin_amdgcn_exp2f(fmaf(score(s, p, 0), sl2, -m_run[qb]));
        const float x1 = __builtin_amdgcn_exp2f(fmaf(score(s, p, 1), sl2, -m_run[qb]));
        const bf16x2 r = {(__bf16)x0, (__bf16)x1};
        if constexpr (LOGS) e_run[qb] += x0 + x1;
        l_run[qb] = __builtin_amdgcn_fdot2_f32_bf16(r, one, l_run[qb], false);
        pf[p / 8][qb][p % 4] = __builtin_bit_cast(uint32_t, r);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bf16x8 vf = ldv(v_slot(t), i);
#pragma unroll
        for (int qb = 0; qb < NQB; ++qb) acc[qb][i % 4] = mfma32(vf, probs(pf, i / 4, qb), acc[qb][i % 4]);
      }
    }
  };

  // Fixed-offset pass first.  Its result stands when every row sum of the work group
  // lies in [2^-60, 2^96] (rows that see no key aside) and every accumulator is finite
  // and below 2^121: then no probability overflowed, and the N keys that
  // underflowed to 0 (logit < -126 in log2 units) weigh at most N 2^-126 against
  // a sum of at least 2^-60.  The accumulator bound leaves room for the merge's sum of
  // up to kSeqMaxSplit = 32 such partials.  Otherwise the group runs the running-max pass.
  bool any_fallback = false;
#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[qb][db] = f32x16{};
    m_run[qb] = 0.f;
    l_run[qb] = 0.f;
  }
  if (nt > 0) {
    any_fallback = !run_fixed();
    if (any_fallback) {
      wait_vmcnt<0>();            // nothing of the abandoned pass is in flight
    } else {
      bool bad = gone;
#pragma unroll
      for (int qb = 0; qb < NQB; ++qb) {
        const float s0 = __shfl(lacc[qb][0], n & 15), s1 = __shfl(lacc[qb][1], n & 15);
        l_run[qb] = n < 16 ? s0 : s1;    // the full row sum, in both lanes of the row
        uint32_t amax = 0;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) amax = max(amax, abs_bits(acc[qb][db][r]));
        bool empty = hi[qb] <= t0 * KT;
        if constexpr (WINDOW) {
          // keys of the range: those of its tiles before and behind the gap
          const int a0 = min(t0, tiles.first) * KT, a1 = min(t0 + nt, tiles.first) * KT;
          const int b0 = (max(t0, tiles.first) + tiles.gap) * KT, b1 = (max(t0 + nt, tiles.first) + tiles.gap) * KT;
          auto meets = [&](int x0, int x1) {
            return (x0 < min(x1, min(min(a.sinks, start[qb]), hi[qb]))) || max(x0, start[qb]) < min(x1, hi[qb]);
          };
          empty = !meets(a0, a1) && !meets(b0, b1);
        }
        bad = bad || !(fixed_offset_ok(l_run[qb], amax) || (empty && __float_as_uint(l_run[qb]) == 0 && amax == 0));
      }
      bad = __any(bad);
      int *flag = reinterpret_cast<int *>(&sK[0][0]);
      __syncthreads();
      if (lane == 0) flag[wave] = bad ? 1 : 0;
      __syncthreads();
      any_fallback = (flag[0] | flag[1]) != 0;
    }
    if (any_fallback) run_max();
  }
  __syncthreads();                // every wave is done with the tiles

#pragma unroll
  for (int qb = 0; qb < NQB; ++qb) {
    const int lrow = wave * 64 + qb * 32 + n;
    // l_run: the row sum of this lane's row (the fixed-offset pass), or this
    // lane's half of it (the running-max pass)
    const float l_tot = any_fallback ? sum_xor32(l_run[qb]) : l_run[qb];
    const float e_tot = LOGS ? sum_xor32(e_run[qb]) : 0.f;
    if (!share.cut) {
      const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot == 0.f ? 0.f : l_tot;
      OutRows<D> out(&sV[0][0] + (wave * 2 + qb) * 32 * D);
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq)
          out.put(n, 8 * db + 2 * rq + g, acc[qb][db][4 * rq] * inv, acc[qb][db][4 * rq + 1] * inv,
                  acc[qb][db][4 * rq + 2] * inv, acc[qb][db][4 * rq + 3] * inv);
      out.store(a, u, head, wave * 64 + qb * 32, lane);
      if constexpr (LOGS) {
        const int row = u.row0 + lrow;
        if (g == 0 && row < u.rows) {
          const int qi = row / a.group, qh = head * a.group + (row - qi * a.group);
          a.lse[(int64_t)qh * a.n_tokens + u.q0 + qi] = log_sum(m_run[qb], e_tot);
        }
      }
    } else {
      float *pp = a.part + share.slot * seq_part_floats(kSeqRows, D, LOGS);
      float *op = pp + (int64_t)lrow * D;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq)
          *reinterpret_cast<f32x4 *>(op + 32 * db + 8 * rq + 4 * g) =
              f32x4{acc[qb][db][4 * rq], acc[qb][db][4 * rq + 1], acc[qb][db][4 * rq + 2], acc[qb][db][4 * rq + 3]};
      if (g == 0) {
        pp[kSeqRows * D + lrow] = l_tot == 0.f ? kMInit : m_run[qb];
        pp[kSeqRows * D + kSeqRows + lrow] = l_tot;
        if constexpr (LOGS) pp[kSeqRows * D + 2 * kSeqRows + lrow] = e_tot;
      }
    }
  }
}

template <bool QUANT>
__global__ __launch_bounds__(128, 1) void seq_attn128_kernel(SeqArgs a) {
  attend128<QUANT ? Keys::kQuant : Keys::kPacked>(a);
}
// With a window: packed tensors, or pages.
template <bool PAGED>
__global__ __launch_bounds__(128, 1) void window_attn128_kernel(SeqArgs a) {
  attend128<PAGED ? Keys::kPaged : Keys::kWindow>(a);
}
// Packed tensors, with the rows' logarithms.
__global__ __launch_bounds__(128, 1) void window_logs128_kernel(SeqArgs a) { attend128<Keys::kWindow, true>(a); }

}  // namespace

hipError_t launch_seq128(const SeqArgs &a, hipStream_t s) {
  const dim3 grid((uint32_t)seq_groups(a)), block(128);
  if (a.cache) hipLaunchKernelGGL((seq_attn128_kernel<true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((seq_attn128_kernel<false>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_window128(const SeqArgs &a, hipStream_t s) {
  const dim3 grid((uint32_t)seq_groups(a)), block(128);
  if (a.table) hipLaunchKernelGGL((window_attn128_kernel<true>), grid, block, 0, s, a);
  else if (a.lse) hipLaunchKernelGGL(window_logs128_kernel, grid, block, 0, s, a);
  else hipLaunchKernelGGL((window_attn128_kernel<false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace hc
