// Gradients of the attention over packed sequences with a window.
#include "hc_mask.h"
#include "hc_window.h"

namespace hc {
namespace {
using namespace dev;

// With P = exp(s q k^T - lse) and dS = P (dO V^T - rowsum(dO O)):
//   dV = P^T dO,  dK = s dS^T Q,  dQ = s dS K.
// Two kernels: one keeps keys and values of a run of keys and walks the queries that see them (dK, dV), the other keeps
// queries and their output gradients and walks their keys (dQ).  Both form the scores again, which is 7 products where
// 5 would do; in return nothing is added up through memory, and the order of every sum is fixed.
//
// Both are one scheme.  A wave keeps two stationary operands B1, B2 (32 columns each, in registers as
// matrix operands) and walks tiles of two streamed tensors A1, A2 (64 rows, in LDS):
//   S = A1 B1 and T = A2 B2 (32 rows x 32 columns), then P and dS from them, and
//   C1 += A^T P or dS with a streamed tensor transposed: for that the LDS is read with the transposing
//   read, 16 lanes fetching 4 rows x 16 dims and each getting 4 rows of one dim.
// Rows are fed to S and T with bits 2 and 3 of their number swapped, so that a lane half g ends up with rows
// 8 g .. 8 g + 7 of every 16 (see hc_device.h), in the order that the second products contract.
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kTile = 64;        // streamed rows of a tile

// Position of 16-byte chunk c of row r of a streamed tile.  Both reads of it want different banks: 16 rows at one
// chunk (a score operand), and 4 neighbouring rows at 64 bytes (a transposing read).
template <int D>
__device__ __forceinline__ int tswz(int r, int c) {
  return c ^ (D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3));
}

// Streamed tiles in LDS: two of each of two tensors.  Addresses are a lane's own part, and constants.
template <int D>
struct Streamed {
  static constexpr int BYTES = kTile * D * 2;
  uint16_t x[2][2][kTile * D];         // [buffer][tensor]
};
using lds8 = const __attribute__((address_space(3))) bf16x8 *;
typedef short s16x4 __attribute__((ext_vector_type(4)));
using ldst = __attribute__((address_space(3))) s16x4 *;

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
  // A operand of a score product: 16 dims kk of rows kperm(n) of the 32 at `tile`
  __device__ __forceinline__ bf16x8 score(uint32_t tile, int kk) const {
    return *(lds8)(uintptr_t)((row ^ (uint32_t)(32 * kk)) + tile);
  }
  // A operand of a second product: dims 32 db .. + 31 of the 16 rows at `tile`
  __device__ __forceinline__ bf16x8 turned(uint32_t tile, int db) const {
    struct { s16x4 a, b; } w;
    w.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)((turn ^ (uint32_t)(64 * db)) + tile));
    w.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)((turn4 ^ (uint32_t)(64 * db)) + tile));
    return __builtin_bit_cast(bf16x8, w);
  }
};

// N DMA instructions (see hc_device.h) behind a wait that covers a base which a vector instruction put into its scalar
// registers just before: 5 wait states, which the compiler does not count for inline assembly.
template <int N>
__device__ __forceinline__ void lds_dma16_settled(const uint16_t *base, const uint32_t (&a)[N], uint32_t lds) {
  static_assert(N == 2 || N == 4, "instructions");
  uint32_t saved;
  if constexpr (N == 2) {
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %4\n\t"
        "s_nop 4\n\t"
        "global_load_lds_dwordx4 %1, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:0x400\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(a[0]), "v"(a[1]), "s"(base), "s"(lds)
        : "memory");
  } else {
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

// Copies a tile to LDS by DMA: rows first .. first + 63 (those behind the last repeat it) of one head.  Instruction j
// of wave w moves 1 KB, the 8 or 4 rows from (N w + j) 512 / D on; a lane fetches the chunk that belongs at its
// 16 bytes.  (The base is 4 KB low, so that no offset goes below zero when 1024 j is taken off.)
template <int D>
struct Copier {
  static constexpr int RW = 512 / D, N = kTile / RW / kWaves;     // rows of an instruction, instructions of a wave
  int lane, wave;
  // p: the tile's first row; left: rows from there on.  (A row's offset stays below 2^31: token strides are below 2^24.)
  __device__ __forceinline__ void copy(const uint16_t *p, int64_t token, int left, uint16_t *tile) const {
    int l = lane;
    asm volatile("" : "+v"(l));      // (the rest is computed at each copy: kept in registers it makes others spill)
    const int row = N * wave * RW + l / (D / 8);
    uint32_t a[N];
#pragma unroll
    for (int j = 0; j < N; ++j)
      a[j] = (uint32_t)min(row + j * RW, left - 1) * (uint32_t)token * 2u +
             (uint32_t)(tswz<D>(row + j * RW, l % (D / 8)) * 16 + 4096 - 1024 * j);
    lds_dma16_settled<N>(p - 2048, a, lds_addr(tile + wave * N * 512));
  }
};

// --- rowsum(dO O), and the logarithms in log2 units -------------------------------------------------
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
    a.stats[at] = a.lse[at] * 1.4426950408889634f;
    a.stats[(int64_t)heads * a.seq.n_tokens + at] = sum;
  }
}

// P and dS of 8 rows as matrix operands
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const bf16x2 r = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, r);
}

// --- dK and dV: a work group takes 128 keys of a key head, each wave 32 --------------------------------
template <int D>
__global__ __launch_bounds__(kThreads, 2) void grad_keys_kernel(GradArgs a) {
  constexpr int NKK = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(1024))) Streamed<D> sT;        // queries, output gradients
  __shared__ __attribute__((aligned(1024))) float sR[2][2][kTile]; // logarithms, rowsum(dO O)
  const SeqArgs &q = a.seq;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const int split = blockIdx.x % a.n_split;
  const int unit = blockIdx.x / a.n_split;
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
  const int first = from(k0), end = max(first, k0 < q.sinks ? u.nq : until(k_last));
  const int nt = (end - first + kTile - 1) / kTile;    // tiles of every query head
  const int64_t items = (int64_t)nt * q.group;
  const int i0 = (int)(items * split / a.n_split), i1 = (int)(items * (split + 1) / a.n_split);
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

  const Copier<D> copier{lane, wave};
  const Reader<D> reader(lane);
  const int64_t plane = (int64_t)q.n_tokens * q.kv_heads * q.group;
  auto load = [&](int item, int b) {
    const int h = head * q.group + item / nt, r0 = first + item % nt * kTile;
    copier.copy(q.q + (u.q0 + r0) * q.q_token + h * q.q_head, q.q_token, u.nq - r0, sT.x[b][0]);
    copier.copy(a.dout + (u.q0 + r0) * a.do_token + h * a.do_head, a.do_token, u.nq - r0, sT.x[b][1]);
    if (wave < 2)
      lds_dma4(a.stats + wave * plane + (int64_t)h * q.n_tokens + u.q0 + r0, u.nq - r0, lane, lds_addr(sR[b][wave]));
  };
  // what this wave has in flight has arrived, and then what every wave had
  auto arrived = [&] {
    wait_vmcnt<0>();
    __syncthreads();
  };
  if (i0 < i1) {
    load(i0, 0);
    arrived();
  }
  const uint32_t tiles = (uint32_t)(uintptr_t)(lvoid)&sT;
  for (int item = i0; item < i1; ++item) {
    const int b = (item - i0) & 1;
    if (item + 1 < i1) load(item + 1, b ^ 1);
    const int r0 = first + item % nt * kTile;
    if (__any(r0 < hi && r0 + kTile > lo)) {
      const bool whole = __all(r0 >= lo && r0 + kTile <= hi);
#pragma unroll 1
      for (int qb = 0; qb < 2; ++qb) {
        const uint32_t tq = tiles + (uint32_t)(b * 2 * Streamed<D>::BYTES + qb * 32 * D * 2), to = tq + Streamed<D>::BYTES;
        f32x16 s = {}, t = {};
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
          s = mfma32(reader.score(tq, kk), kf[kk], s);
          t = mfma32(reader.score(to, kk), vf[kk], t);
        }
        u32x4 pf[2], df[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int at = 32 * qb + 16 * c + 8 * g;         // the 8 rows of this lane
          float p[8], d[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(s[8 * c + e], q.scale_log2, -sR[b][0][at + e]));
          if (!whole)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int i = r0 + at + e;
              if ((i < lo) | (i >= hi)) p[e] = 0.f;
            }
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = p[e] * (t[8 * c + e] - sR[b][1][at + e]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pf[c][e] = pack2(p[2 * e], p[2 * e + 1]);
            df[c][e] = pack2(d[2 * e], d[2 * e + 1]);
          }
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            dv[db] = mfma32(reader.turned(to + (uint32_t)(c * 16 * D * 2), db), __builtin_bit_cast(bf16x8, pf[c]), dv[db]);
            dk[db] = mfma32(reader.turned(tq + (uint32_t)(c * 16 * D * 2), db), __builtin_bit_cast(bf16x8, df[c]), dk[db]);
          }
      }
    }
    if (item + 1 < i1) arrived();
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
__global__ __launch_bounds__(kThreads, 2) void grad_queries_kernel(GradArgs a) {
  constexpr int NKK = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(1024))) Streamed<D> sT;        // keys, values
  SeqArgs q = a.seq;
  const int group = q.group;
  q.group = 1;                       // rows are the queries of one head
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const int heads = q.kv_heads * group;
  const int tile = __builtin_amdgcn_readfirstlane((int)blockIdx.x / heads), h = (int)blockIdx.x - tile * heads, head = h / group;
  SeqUnit u;
  if (!seq_unit<kSeqRows>(q, tile, u)) return;
  const int row = u.row0 + 32 * wave + n, at = min(row, u.nq - 1);
  const Seen mine = seen_by(q, u, at);
  const KeyTiles tiles(seen_by(q, u, u.row0), seen_by(q, u, min(u.row0 + kSeqRows, u.nq) - 1));
  bf16x8 qf[NKK], of[NKK];
  {
    const uint16_t *qp = q.q + (u.q0 + at) * q.q_token + h * q.q_head + 8 * g;
    const uint16_t *op = a.dout + (u.q0 + at) * a.do_token + h * a.do_head + 8 * g;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) {
      qf[kk] = ld_g16(qp + 16 * kk);
      of[kk] = ld_g16(op + 16 * kk);
    }
  }
  const float *sp = a.stats + (int64_t)h * q.n_tokens + u.q0 + at;
  const float lse = sp[0], delta = sp[(int64_t)q.n_tokens * heads];
  f32x16 dq[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dq[db] = f32x16{};
  const Copier<D> copier{lane, wave};
  const Reader<D> reader(lane);
  const uint16_t *kp = q.k + u.k0 * q.k_token + head * q.k_head, *vp = q.v + u.k0 * q.v_token + head * q.v_head;
  auto load = [&](int t, int b) {
    const int64_t at = (int64_t)tiles.place(t) * kTile;
    copier.copy(kp + at * q.k_token, q.k_token, u.nk - (int)at, sT.x[b][0]);
    copier.copy(vp + at * q.v_token, q.v_token, u.nk - (int)at, sT.x[b][1]);
  };
  auto arrived = [&] {
    wait_vmcnt<0>();
    __syncthreads();
  };
  if (tiles.n > 0) {
    load(0, 0);
    arrived();
  }
  const uint32_t base = (uint32_t)(uintptr_t)(lvoid)&sT;
  for (int t = 0; t < tiles.n; ++t) {
    const int b = t & 1, place = tiles.place(t);
    if (t + 1 < tiles.n) load(t + 1, b ^ 1);
    const bool whole = tiles.whole(place, q.sinks);
#pragma unroll 1
    for (int kb = 0; kb < 2; ++kb) {
      const uint32_t tk = base + (uint32_t)(b * 2 * Streamed<D>::BYTES + kb * 32 * D * 2), tv = tk + Streamed<D>::BYTES;
      f32x16 s = {}, d = {};
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        s = mfma32(reader.score(tk, kk), qf[kk], s);
        d = mfma32(reader.score(tv, kk), of[kk], d);
      }
      u32x4 df[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[8 * c + e], q.scale_log2, -lse));
          x[e] = p * (d[8 * c + e] - delta);
        }
        if (!whole)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!mine.sees(place * kTile + 32 * kb + 16 * c + 8 * g + e)) x[e] = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) df[c][e] = pack2(x[2 * e], x[2 * e + 1]);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
          dq[db] = mfma32(reader.turned(tk + (uint32_t)(c * 16 * D * 2), db), __builtin_bit_cast(bf16x8, df[c]), dq[db]);
    }
    if (t + 1 < tiles.n) arrived();
  }
  if (row >= u.nq) return;
  uint16_t *op = a.dq + (u.q0 + row) * a.dq_token + h * a.dq_head;
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      uint2 w;
      w.x = pack2(dq[db][4 * rq] * a.scale, dq[db][4 * rq + 1] * a.scale);
      w.y = pack2(dq[db][4 * rq + 2] * a.scale, dq[db][4 * rq + 3] * a.scale);
      *reinterpret_cast<uint2 *>(op + 32 * db + 8 * rq + 4 * g) = w;
    }
}

template <int D>
hipError_t launch(const GradArgs &a, hipStream_t s) {
  const int heads = a.seq.kv_heads * a.seq.group;
  const int64_t rows = (int64_t)a.seq.n_tokens * heads * (D / 8);
  if (rows > 0) hipLaunchKernelGGL(grad_stats_kernel<D>, dim3((uint32_t)((rows + 255) / 256)), dim3(256), 0, s, a);
  if (a.key_tiles > 0) {
    hipLaunchKernelGGL(grad_keys_kernel<D>, dim3((uint32_t)(a.key_tiles * a.seq.kv_heads * a.n_split)), dim3(kThreads), 0, s, a);
    if (a.n_split > 1)
      hipLaunchKernelGGL(grad_merge_kernel<D>, dim3((uint32_t)(a.key_tiles * a.seq.kv_heads * (kGradKeys * D / 1024))), dim3(256), 0, s, a);
  }
  if (a.seq.tiles > 0)
    hipLaunchKernelGGL(grad_queries_kernel<D>, dim3((uint32_t)(a.seq.tiles * heads)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grad(const GradArgs &a, int head_dim, hipStream_t s) {
  return head_dim == 128 ? launch<128>(a, s) : launch<64>(a, s);
}

}  // namespace hc
