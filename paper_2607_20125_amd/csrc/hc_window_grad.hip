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

// What a row needs besides its dims: the logarithm of its sum in log2 units, rowsum(dO O), and its keys.
struct RowStats {
  float lse[kTile], delta[kTile];
  int end[kTile], start[kTile];
};

template <int D>
struct Streamed {
  uint16_t x[kTile * D];
  // A operand of a score product: 16 dims kk of row kperm(n) of 32-row block b
  __device__ __forceinline__ bf16x8 row(int b, int kk, int n, int g) const {
    const int r = 32 * b + kperm(n);
    return *reinterpret_cast<const bf16x8 *>(&x[r * D + tswz<D>(r, 2 * kk + g) * 8]);
  }
  // A operand of a second product: dims 32 db .. + 31 of rows 16 c .. + 15
  __device__ __forceinline__ bf16x8 turned(int c, int db, int lane) const {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    using ldst = __attribute__((address_space(3))) s16x4 *;
    const int gl = lane >> 4, i = lane & 15;
    const int r = 16 * c + 8 * (gl / 2) + i / 4, chunk = 4 * db + 2 * (gl % 2) + (i % 4) / 2;
    const uint32_t base = (uint32_t)(uintptr_t)(lvoid)x;
    const uint32_t at = base + (uint32_t)(r * D + tswz<D>(r, chunk) * 8 + (i % 2) * 4) * 2;
    const uint32_t at4 = base + (uint32_t)((r + 4) * D + tswz<D>(r + 4, chunk) * 8 + (i % 2) * 4) * 2;
    struct { s16x4 a, b; } w;
    w.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)at);
    w.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ldst)(uintptr_t)at4);
    return __builtin_bit_cast(bf16x8, w);
  }
};

// A tile on its way: rows first .. first + 63 (those behind the last repeat it) of one head.
template <int D>
struct Loader {
  static constexpr int N = kTile * D / 8 / kThreads;     // 16-byte pieces of a thread
  u32x4 w[N];
  __device__ __forceinline__ void load(const uint16_t *p, int64_t token, int first, int last) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = threadIdx.x + i * kThreads;
      w[i] = gld16(p + min(first + c / (D / 8), last) * token + (c % (D / 8)) * 8);
    }
  }
  __device__ __forceinline__ void put(Streamed<D> &t) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = threadIdx.x + i * kThreads, r = c / (D / 8);
      *reinterpret_cast<u32x4 *>(&t.x[r * D + tswz<D>(r, c % (D / 8)) * 8]) = w[i];
    }
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
    a.stats[2 * at] = a.lse[at] * 1.4426950408889634f;
    a.stats[2 * at + 1] = sum;
  }
}

// P and dS of 8 rows as matrix operands
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const bf16x2 r = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, r);
}

// --- dK and dV: a work group takes 128 keys of a key head, each wave 32 --------------------------------
template <int D>
__global__ __launch_bounds__(kThreads, 1) void grad_keys_kernel(GradArgs a) {
  constexpr int NKK = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(1024))) Streamed<D> sQ[2];
  __shared__ __attribute__((aligned(1024))) Streamed<D> sO[2];
  __shared__ RowStats sR[2];
  const SeqArgs &q = a.seq;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const int split = blockIdx.x % a.n_split;
  const int unit = blockIdx.x / a.n_split;
  const int tile = __builtin_amdgcn_readfirstlane(unit / q.kv_heads), head = unit - tile * q.kv_heads;
  SeqUnit u;
  if (!seq_unit<kGradKeys, true>(q, tile, u)) return;
  const int k0 = u.row0, k_last = min(k0 + kGradKeys, u.nk) - 1;

  // the queries that see any of the keys
  int first = 0, end = u.nq;
  if (q.block) {
    const int64_t off = (int64_t)u.nk - u.nq;          // position of query 0
    first = (int)min(max((int64_t)(k0 / q.block) * q.block - off, (int64_t)0), (int64_t)u.nq);
    if (q.window && k0 >= q.sinks)
      end = (int)min(max(((int64_t)k_last + q.window) / q.block * q.block - off, (int64_t)first), (int64_t)u.nq);
  }
  const int nt = (end - first + kTile - 1) / kTile;    // of every query head
  const int64_t items = (int64_t)nt * q.group;
  const int i0 = (int)(items * split / a.n_split), i1 = (int)(items * (split + 1) / a.n_split);

  const int key = k0 + 32 * wave + n;
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

  Loader<D> lq, lo;
  float2 st = {0.f, 0.f};
  Seen seen{};
  auto load = [&](int item) {
    const int h = head * q.group + item / nt, r0 = first + item % nt * kTile;
    lq.load(q.q + u.q0 * q.q_token + h * q.q_head, q.q_token, r0, u.nq - 1);
    lo.load(a.dout + u.q0 * a.do_token + h * a.do_head, a.do_token, r0, u.nq - 1);
    if (tid < kTile) {
      const int i = r0 + tid;
      seen = i < u.nq ? seen_by(q, u, i) : Seen{0, 0, 0};
      st = *(const float2 *)(a.stats + 2 * ((int64_t)h * q.n_tokens + u.q0 + min(i, u.nq - 1)));
    }
  };
  auto put = [&](int b) {
    lq.put(sQ[b]);
    lo.put(sO[b]);
    if (tid < kTile) {
      sR[b].lse[tid] = st.x;
      sR[b].delta[tid] = st.y;
      sR[b].end[tid] = seen.end;
      sR[b].start[tid] = seen.start;
    }
  };
  if (i0 < i1) {
    load(i0);
    put(0);
    __syncthreads();
  }
  for (int item = i0; item < i1; ++item) {
    const int b = (item - i0) & 1;
    if (item + 1 < i1) load(item + 1);
    const int r0 = first + item % nt * kTile;
    const int wk0 = k0 + 32 * wave, wk1 = min(wk0 + 31, u.nk - 1);
    const Seen lo_seen = seen_by(q, u, r0), hi_seen = seen_by(q, u, min(r0 + kTile, u.nq) - 1);
    const bool any = wk0 <= k_last && wk0 < hi_seen.end && (wk0 < q.sinks || wk1 >= lo_seen.start);
    const bool whole = r0 + kTile <= u.nq && wk1 < lo_seen.end && (wk1 < q.sinks || wk0 >= hi_seen.start);
    if (any) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        f32x16 s = {}, t = {};
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
          s = mfma32(sQ[b].row(qb, kk, n, g), kf[kk], s);
          t = mfma32(sO[b].row(qb, kk, n, g), vf[kk], t);
        }
        u32x4 pf[2], df[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int at = 32 * qb + 16 * c + 8 * g;         // the 8 rows of this lane
          float p[8], d[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(fmaf(s[8 * c + e], q.scale_log2, -sR[b].lse[at + e]));
            if (!whole) {
              const int x = sR[b].end[at + e], y = sR[b].start[at + e];
              if (!(key < x && (key < q.sinks || key >= y))) p[e] = 0.f;
            }
            d[e] = p[e] * (t[8 * c + e] - sR[b].delta[at + e]);
          }
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
            dv[db] = mfma32(sO[b].turned(2 * qb + c, db, lane), __builtin_bit_cast(bf16x8, pf[c]), dv[db]);
            dk[db] = mfma32(sQ[b].turned(2 * qb + c, db, lane), __builtin_bit_cast(bf16x8, df[c]), dk[db]);
          }
      }
    }
    if (item + 1 < i1) {
      put(b ^ 1);
      __syncthreads();
    }
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
__global__ __launch_bounds__(kThreads, 1) void grad_queries_kernel(GradArgs a) {
  constexpr int NKK = D / 16, NDB = D / 32;
  __shared__ __attribute__((aligned(1024))) Streamed<D> sK[2];
  __shared__ __attribute__((aligned(1024))) Streamed<D> sV[2];
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
  const float2 st = *(const float2 *)(a.stats + 2 * ((int64_t)h * q.n_tokens + u.q0 + at));
  f32x16 dq[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) dq[db] = f32x16{};
  Loader<D> lk, lv;
  const uint16_t *kp = q.k + u.k0 * q.k_token + head * q.k_head, *vp = q.v + u.k0 * q.v_token + head * q.v_head;
  auto load = [&](int t) {
    lk.load(kp, q.k_token, tiles.place(t) * kTile, u.nk - 1);
    lv.load(vp, q.v_token, tiles.place(t) * kTile, u.nk - 1);
  };
  if (tiles.n > 0) {
    load(0);
    lk.put(sK[0]);
    lv.put(sV[0]);
    __syncthreads();
  }
  for (int t = 0; t < tiles.n; ++t) {
    const int b = t & 1, place = tiles.place(t);
    if (t + 1 < tiles.n) load(t + 1);
    const bool whole = tiles.whole(place, q.sinks);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s = {}, d = {};
#pragma unroll
      for (int kk = 0; kk < NKK; ++kk) {
        s = mfma32(sK[b].row(kb, kk, n, g), qf[kk], s);
        d = mfma32(sV[b].row(kb, kk, n, g), of[kk], d);
      }
      u32x4 df[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float p = __builtin_amdgcn_exp2f(fmaf(s[8 * c + e], q.scale_log2, -st.x));
          if (!whole && !mine.sees(place * kTile + 32 * kb + 16 * c + 8 * g + e)) p = 0.f;
          x[e] = p * (d[8 * c + e] - st.y);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) df[c][e] = pack2(x[2 * e], x[2 * e + 1]);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
          dq[db] = mfma32(sK[b].turned(2 * kb + c, db, lane), __builtin_bit_cast(bf16x8, df[c]), dq[db]);
    }
    if (t + 1 < tiles.n) {
      lk.put(sK[b ^ 1]);
      lv.put(sV[b ^ 1]);
      __syncthreads();
    }
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
