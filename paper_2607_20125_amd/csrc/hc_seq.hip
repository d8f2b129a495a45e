// Attention over sequences: packed keys and values in bf16, or the 4-bit cache; and
// the merge of partial results.
#include "hc_seq.h"

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// One work group: 128 rows (queries times query heads of one key head) of a
// sequence on 4 waves of 32, over the key tiles of its range, 64 keys each.  Tiles go
// global -> registers -> LDS: the loads of tile t + 1 are issued before the products of
// tile t, and are converted (4-bit codes) and transposed (V) on their way into the
// other LDS buffer.  Online softmax with lazy rescaling; layouts as in hc_device.h.  Probabilities are
// rounded to bf16, the operand type of the product with V (wider types run at a fraction of its rate); the row sums
// add the rounded ones, so that the weights in use add up to 1.  Outputs are 1.1 to 1.4 times as far from 64
// bits as with probabilities in 32 (two blocks over their text 0.0023 and 0.0017 of their size).  Two work groups
// (three with 64-dim heads: 5% faster where they fill the card) share a CU, a wave each on every SIMD, and hide each
// other's loads and barriers.  (With S(t+1) computed beside
// the softmax of tile t, as the dense kernels do, 128-dim heads need more than the 256 registers
// and 64-dim heads gain nothing.)  Measured: two 480P blocks over 226 and 513 keys of text
// (12 heads of 128 dims) 42 us, half of it for queries in and outputs out; 9360 rows of 12 heads of 64 dims
// over 4096 keys 200 us, 0.59 PFLOP/s: exponentials, sums and conversions and the products take
// turns on a SIMD (vector units busy 60%, matrix cores 27%).
// ---------------------------------------------------------------------------
constexpr int kWaves = kSeqRows / 32;

template <int D, bool QUANT>
__global__ __launch_bounds__(64 * kWaves, D == 64 ? 3 : 2) void seq_attn_kernel(SeqArgs a) {
  constexpr int KT = kSeqKeys, NKK = D / 16, NDB = D / 32, TILE = KT * D;
  constexpr int NT = 64 * kWaves;
  __shared__ __attribute__((aligned(1024))) uint16_t sK[2][TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sV[2][TILE];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, g = lane >> 5;
  const SeqShare share = seq_share(a);
  const int head = share.head;
  SeqUnit u;
  if (!seq_unit<kSeqRows>(a, share.tile, u)) return no_unit(share);

  // this lane's row, and its query and head
  const int row = u.row0 + wave * 32 + n;
  const int at = min(row, u.rows - 1);
  const int qi = at / a.group, qh = head * a.group + (at - qi * a.group);
  bf16x8 qf[NKK];
  {
    const uint16_t *qp = a.q + (u.q0 + qi) * a.q_token + qh * a.q_head;
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk) qf[kk] = ld_g16(qp + 16 * kk + 8 * g);
  }
  const int hi = seen_keys(a, u, qi);
  // keys that every row of the unit sees, and that any row sees (seen_keys grows with the query)
  const int first = u.row0 / a.group, last = min(u.row0 + kSeqRows, u.rows) - 1;
  const int lo_all = seen_keys(a, u, first), hi_all = seen_keys(a, u, last / a.group);
  const int nt_all = (hi_all + KT - 1) / KT;
  int t0, t1;
  key_range(a, u, share, nt_all, t0, t1);
  const float sl2 = a.scale_log2;

  // --- tiles ---------------------------------------------------------------------
  // K: chunk c (8 dims) of key r goes to LDS row kperm(r), position kswz.  V: 8 keys of
  // one dim are 16 bytes ([group of 8 keys][d][8]); dim d of a group is kept at d ^ (d / 16 % 4), so that
  // 16 lanes that write 4 dims each reach all banks with each of them.
  constexpr int KI = QUANT ? 1 : TILE / 8 / NT;      // K loads of a thread
  u32x4 kr[KI], vr[QUANT ? 1 : 4];
  uint32_t ks = 0, vs[2] = {0, 0};
  const uint8_t *cbase = QUANT ? a.cache + ((int64_t)u.seq * a.kv_heads + head) * a.cache_head : nullptr;
  const uint16_t *kbase = QUANT ? nullptr : a.k + u.k0 * a.k_token + head * a.k_head;
  const uint16_t *vbase = QUANT ? nullptr : a.v + u.k0 * a.v_token + head * a.v_head;
  // 4-bit tiles: thread -> (token, 32 dims) of K and (8 tokens, 4 dims) of V; with 64-dim
  // heads half the threads take K and half V
  constexpr int NG = D / kQGroup;
  const bool has_k = !QUANT || D == 128 || tid < NT / 2;
  const bool has_v = D == 128 || (QUANT ? tid >= NT / 2 : tid < NT / 2);
  const int ki = tid % (KT * NG), vi = tid % (8 * D / 4);
  const int k_tok = ki / NG, k_grp = ki % NG;
  const int v_grp = vi / (D / 4), v_dim = vi % (D / 4) * 4;

  auto load = [&](int t) {
    if constexpr (QUANT) {
      const uint8_t *tp = cbase + (int64_t)t * qtile_bytes(D);
      if (has_k) {
        kr[0] = *(gptr16)(tp + ki * 16);
        ks = tp[qtile_k_scales(D) + ki];
      }
      if (has_v) {
        vr[0] = *(gptr16)(tp + qtile_v(D) + vi * 16);
        const uint32_t *sp = (const uint32_t *)(tp + qtile_v_scales(D) + (v_grp * NG + v_dim / kQGroup) * 8);
        vs[0] = sp[0];
        vs[1] = sp[1];
      }
    } else {
      const int k00 = t * KT;
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int c = tid + i * NT;
        const int key = min(k00 + c / (D / 8), u.nk - 1);
        kr[i] = gld16(kbase + key * a.k_token + (c % (D / 8)) * 8);
      }
      if (has_v) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = min(k00 + 8 * v_grp + i, u.nk - 1);
          const uint2 w = *(const uint2 *)(vbase + key * a.v_token + v_dim);
          vr[i / 2][2 * (i % 2)] = w.x;
          vr[i / 2][2 * (i % 2) + 1] = w.y;
        }
      }
    }
  };
  auto put_k = [&](int b, int key, int c, u32x4 w) {
    const int r = (key & ~31) | kperm(key & 31);
    *reinterpret_cast<u32x4 *>(&sK[b][r * D + kswz<D>(r, c) * 8]) = w;
  };
  // dims 2 i, 2 i + 1 of tokens 2 j (x) and 2 j + 1 (y) become words of two tokens
  auto low2 = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); };
  auto high2 = [](uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); };
  auto put_v_dim = [&](int b, int e, u32x4 w) {
    const int dim = v_dim + e;
    *reinterpret_cast<u32x4 *>(&sV[b][(v_grp * D + (dim ^ (dim >> 4 & 3))) * 8]) = w;
  };
  auto put = [&](int t) {
    const int b = t & 1;
    if constexpr (QUANT) {
      if (has_k) {
        const float scale = __uint_as_float(ks << 23);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const uint32_t w = kr[0][m];
          put_k(b, k_tok, 4 * k_grp + m,
                u32x4{values2<0>(w, scale), values2<1>(w, scale), values2<2>(w, scale), values2<3>(w, scale)});
        }
      }
      if (has_v) {
        // slots behind the end hold anything: their scale becomes the smallest, so that
        // a probability of 0 times their value is 0
        const int left = u.nk - t * KT - 8 * v_grp;
        uint32_t s0 = vs[0], s1 = vs[1];
        if (left < 8) {
          s0 = left >= 4 ? s0 : left <= 0 ? 0u : s0 & ((1u << (8 * left)) - 1u);
          s1 = left <= 4 ? 0u : s1 & ((1u << (8 * (left - 4))) - 1u);
        }
        u32x4 d[4];
        auto two = [&](int j, uint32_t w, float sx, float sy) {    // tokens 2 j and 2 j + 1
          const uint32_t x0 = values2<0>(w, sx), x1 = values2<1>(w, sx);
          const uint32_t y0 = values2<2>(w, sy), y1 = values2<3>(w, sy);
          d[0][j] = low2(x0, y0);
          d[1][j] = high2(x0, y0);
          d[2][j] = low2(x1, y1);
          d[3][j] = high2(x1, y1);
        };
        two(0, vr[0][0], scale_of<0>(s0), scale_of<1>(s0));
        two(1, vr[0][1], scale_of<2>(s0), scale_of<3>(s0));
        two(2, vr[0][2], scale_of<0>(s1), scale_of<1>(s1));
        two(3, vr[0][3], scale_of<2>(s1), scale_of<3>(s1));
#pragma unroll
        for (int e = 0; e < 4; ++e) put_v_dim(b, e, d[e]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < KI; ++i) {
        const int c = tid + i * NT;
        put_k(b, c / (D / 8), c % (D / 8), kr[i]);
      }
      if (has_v) {
        u32x4 d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          d[0][j] = low2(vr[j][0], vr[j][2]);
          d[1][j] = high2(vr[j][0], vr[j][2]);
          d[2][j] = low2(vr[j][1], vr[j][3]);
          d[3][j] = high2(vr[j][1], vr[j][3]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) put_v_dim(b, e, d[e]);
      }
    }
  };

  // --- key loop -------------------------------------------------------------------
  f32x16 acc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db) acc[db] = f32x16{};
  float m_run = kMInit, l_run = 0.f;
  if (t0 < t1) {
    load(t0);
    put(t0);
    __syncthreads();
  }
  for (int t = t0; t < t1; ++t) {
    const int b = t & 1;
    if (t + 1 < t1) load(t + 1);
    f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
    for (int kk = 0; kk < NKK; ++kk)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(
            &sK[b][(32 * kb + n) * D + kswz<D>(32 * kb + n, 2 * kk + g) * 8]);
        s[kb] = mfma32(kf, qf[kk], s[kb]);
      }
    if ((t + 1) * KT > lo_all) {
      const int rem = hi - t * KT;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + kperm(8 * (r >> 2) + 4 * g + (r & 3)) >= rem) s[kb][r] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = larger(mx, larger(s[0][r], s[1][r]));
    mx = larger_xor32(mx) * sl2;
    if (__any(mx > m_run + kRescale)) {
      const float m_new = larger(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db) acc[db] *= alpha;
    }
    bf16x8 pf[2][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          pf[kb][h][e] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[kb][8 * h + e], sl2, -m_run));
        const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          l_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[kb][h][e], pf[kb][h][e + 1]}, one, l_run, false);
      }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          const int dim = 32 * db + n;
          const bf16x8 vf =
              *reinterpret_cast<const bf16x8 *>(&sV[b][((4 * kb + 2 * h + g) * D + (dim ^ (dim >> 4 & 3))) * 8]);
          acc[db] = mfma32(vf, pf[kb][h], acc[db]);
        }
    if (t + 1 < t1) {
      put(t + 1);
      __syncthreads();
    }
  }

  const float l_tot = sum_xor32(l_run);
  if (!share.cut) {
    const float inv = l_tot > 0.f ? 1.f / l_tot : l_tot == 0.f ? 0.f : l_tot;
    __syncthreads();              // every wave is done with the tiles
    OutRows<D> out(&sK[0][0] + wave * 32 * D);
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq)
        out.put(n, 8 * db + 2 * rq + g, acc[db][4 * rq] * inv, acc[db][4 * rq + 1] * inv, acc[db][4 * rq + 2] * inv,
                acc[db][4 * rq + 3] * inv);
    out.store(a, u, head, wave * 32, lane);
  } else {
    const int lrow = wave * 32 + n;
    float *pp = a.part + share.slot * seq_part_floats(kSeqRows, D);
    float *op = pp + (int64_t)lrow * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq)
        *reinterpret_cast<f32x4 *>(op + 32 * db + 8 * rq + 4 * g) =
            f32x4{acc[db][4 * rq], acc[db][4 * rq + 1], acc[db][4 * rq + 2], acc[db][4 * rq + 3]};
    if (g == 0) {
      pp[kSeqRows * D + lrow] = m_run;
      pp[kSeqRows * D + kSeqRows + lrow] = l_tot;
    }
  }
}

// ---------------------------------------------------------------------------
// Merge of the n_split partial results of every unit: O = sum_i 2^(m_i - M) acc_i /
// sum_i 2^(m_i - M) l_i.  A thread takes 4 dims of a row; a work group 256 * 4 / D rows.
// ---------------------------------------------------------------------------
template <int D, int R>
__global__ __launch_bounds__(256) void seq_merge_kernel(SeqArgs a) {
  constexpr int TR = D / 4, RW = 256 / TR, RP = R / RW;      // threads a row, rows a group, groups a unit
  static_assert(R % RW == 0, "rows of a unit");
  const int unit = blockIdx.x / RP;
  SeqUnit u;
  int head;
  if (!left_unit(a, unit, u, head)) return;
  const int lrow = (blockIdx.x % RP) * RW + threadIdx.x / TR, row = u.row0 + lrow;
  if (row >= u.rows) return;
  const int dim = threadIdx.x % TR * 4;
  const float *pp = a.part + (int64_t)unit * a.n_split * seq_part_floats(R, D);
  float M = kMInit;
  for (int i = 0; i < a.n_split; ++i) M = fmaxf(M, pp[i * seq_part_floats(R, D) + R * D + lrow]);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  for (int i = 0; i < a.n_split; ++i) {
    const float *p = pp + i * seq_part_floats(R, D);
    const float w = __builtin_amdgcn_exp2f(p[R * D + lrow] - M);
    l += w * p[R * D + R + lrow];
    o += w * *reinterpret_cast<const f32x4 *>(p + lrow * D + dim);
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  const int qi = row / a.group, qh = head * a.group + (row - qi * a.group);
  const bf16x2 x = {(__bf16)(o[0] * inv), (__bf16)(o[1] * inv)}, y = {(__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
  uint2 w;
  w.x = __builtin_bit_cast(uint32_t, x);
  w.y = __builtin_bit_cast(uint32_t, y);
  *reinterpret_cast<uint2 *>(a.o + (u.q0 + qi) * a.o_token + qh * a.o_head + dim) = w;
}

// The same for many partial results: a work group takes one row, its threads 4 dims of every
// 256 * 4 / D-th of them, so that their reads are in flight together.  (One thread summing all 128
// of a long cache's row took 66 us beside an attention kernel of 29.)
template <int D, int R>
__global__ __launch_bounds__(256) void seq_merge_many_kernel(SeqArgs a) {
  constexpr int TR = D / 4, NG = 256 / TR;
  __shared__ float sW[kDecodeMaxSplit], sL[kDecodeMaxSplit], sO[NG][D], sM[4];
  const int unit = blockIdx.x / R, lrow = blockIdx.x % R;
  SeqUnit u;
  int head;
  if (!left_unit(a, unit, u, head)) return;
  const int row = u.row0 + lrow;
  if (row >= u.rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float *pp = a.part + (int64_t)unit * a.n_split * seq_part_floats(R, D);
  const float *ml = pp + tid * seq_part_floats(R, D) + R * D + lrow;
  const float m = tid < a.n_split ? ml[0] : kMInit;
  const float l = tid < a.n_split ? ml[R] : 0.f;
  float M = m;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) M = fmaxf(M, __shfl_xor(M, d));
  if (lane == 0) sM[wave] = M;
  __syncthreads();
  M = fmaxf(fmaxf(sM[0], sM[1]), fmaxf(sM[2], sM[3]));
  const float w = __builtin_amdgcn_exp2f(m - M);
  sW[tid] = w;
  sL[tid] = w * l;
  __syncthreads();
  const int grp = tid / TR, dim = tid % TR * 4;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const float *op = pp + lrow * D + dim;
#pragma unroll 4
  for (int i = grp; i < a.n_split; i += NG)
    o += sW[i] * *reinterpret_cast<const f32x4 *>(op + i * seq_part_floats(R, D));
  *reinterpret_cast<f32x4 *>(&sO[grp][dim]) = o;
  __syncthreads();
  if (tid >= TR) return;
  float total = 0.f;
  for (int i = 0; i < a.n_split; ++i) total += sL[i];
#pragma unroll
  for (int k = 1; k < NG; ++k) o += *reinterpret_cast<const f32x4 *>(&sO[k][dim]);
  const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
  const int qi = row / a.group, qh = head * a.group + (row - qi * a.group);
  const bf16x2 x = {(__bf16)(o[0] * inv), (__bf16)(o[1] * inv)}, y = {(__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
  uint2 r;
  r.x = __builtin_bit_cast(uint32_t, x);
  r.y = __builtin_bit_cast(uint32_t, y);
  *reinterpret_cast<uint2 *>(a.o + (u.q0 + qi) * a.o_token + qh * a.o_head + dim) = r;
}

}  // namespace

hipError_t launch_seq(const SeqArgs &a, int head_dim, hipStream_t s) {
  const dim3 grid((uint32_t)seq_groups(a)), block(64 * kWaves);
  if (head_dim == 128 && a.wide) return launch_seq128(a, s);
  if (head_dim == 128) {
    if (a.cache) hipLaunchKernelGGL((seq_attn_kernel<128, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((seq_attn_kernel<128, false>), grid, block, 0, s, a);
  } else {
    if (a.cache) hipLaunchKernelGGL((seq_attn_kernel<64, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((seq_attn_kernel<64, false>), grid, block, 0, s, a);
  }
  return hipGetLastError();
}

hipError_t launch_seq_merge(const SeqArgs &a, int head_dim, int rows, hipStream_t s) {
  const bool many = a.n_split > 8;
  const int per = many ? rows : rows * head_dim / 1024;      // work groups of a unit
  const dim3 grid((uint32_t)(seq_cut_units(a) * per)), block(256);
#define HC_MERGE(D, R)                                                                     \
  if (many) hipLaunchKernelGGL((seq_merge_many_kernel<D, R>), grid, block, 0, s, a);       \
  else hipLaunchKernelGGL((seq_merge_kernel<D, R>), grid, block, 0, s, a)
  if (head_dim == 128) {
    if (rows == kSeqRows) { HC_MERGE(128, kSeqRows); }
    else { HC_MERGE(128, kDecodeRows); }
  } else {
    if (rows == kSeqRows) { HC_MERGE(64, kSeqRows); }
    else { HC_MERGE(64, kDecodeRows); }
  }
#undef HC_MERGE
  return hipGetLastError();
}

}  // namespace hc
