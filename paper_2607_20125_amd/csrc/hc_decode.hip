// Attention over the 4-bit cache for few rows per sequence (single tokens).
#include "hc_seq.h"

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// One work group: up to 16 rows (queries times query heads of one key head) of a
// sequence over one range of its key tiles; its 4 waves take every fourth tile and are
// merged in LDS at the end.
//
// Bound by the cache's bytes: 17 per 32 values.  Nothing is shared between waves, so a
// tile goes from memory to registers (one tile ahead), is converted there and is an
// operand of the matrix cores without passing LDS:
//  * S^T = K Q^T with 16x16x32 products.  A lane's 16 bytes (8 with 64-dim heads) are
//    consecutive dims of one key; the dims are contracted in that order, with Q read to match.
//    Key rows are fed so that lane group g ends up with keys 8 g .. 8 g + 7 of every 32.
//  * O^T = V^T P^T then needs 8 keys of one dim: the cache keeps V in groups of 8 tokens,
//    and pairs of converted words give pairs of tokens by one byte permute each.  The probabilities are
//    rounded to bf16 for it, and their sum is of the rounded ones (see hc_seq.hip).
// Measured: 8 key heads of 131072 tokens (143 MB) 26.5 us, 5.4 TB/s, and 4 for the merge; 48 sequences of 1 to 8192
// tokens with 64-dim heads (52 MB) 20.7 us, where work groups of a few microseconds end unevenly.
// A second tile ahead, or registers capped for more waves, spills.
// ---------------------------------------------------------------------------
constexpr int kWaves = 4;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// With the value 16 lanes away (the other half of a 32-lane row).
__device__ __forceinline__ float larger_xor16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return larger(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_xor16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void decode_attn_kernel(SeqArgs a) {
  constexpr int R = kDecodeRows, KT = kSeqKeys;
  constexpr int NM = D / 32;             // score products per 16 keys; words of a lane's K piece
  constexpr int NV = D / 16;             // output products per 32 keys; dims of a lane's V piece
  constexpr int NG = D / kQGroup;
  __shared__ float sO[kWaves][R][D + 4];
  __shared__ float sM[kWaves][R], sL[kWaves][R];

  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, g = lane >> 4;
  const SeqShare share = seq_share(a);
  const int head = share.head;
  SeqUnit u;
  if (!seq_unit<R>(a, share.tile, u)) return no_unit(share);

  const int at = min(u.row0 + i, u.rows - 1);
  const int qi = at / a.group, qh = head * a.group + (at - qi * a.group);
  bf16x8 qf[NM];
  {
    const uint16_t *qp = a.q + (u.q0 + qi) * a.q_token + qh * a.q_head + g * (D / 4);
#pragma unroll
    for (int m = 0; m < NM; ++m) qf[m] = ld_g16(qp + 8 * m);
  }
  const int hi = seen_keys(a, u, qi);
  const int last = min(u.row0 + R, u.rows) - 1;
  const int lo_all = seen_keys(a, u, u.row0 / a.group), hi_all = seen_keys(a, u, last / a.group);
  const int nt_all = (hi_all + KT - 1) / KT;
  int t0, t1;
  key_range(a, u, share, nt_all, t0, t1);
  const float sl2 = a.scale_log2;
  const uint8_t *base = a.cache + ((int64_t)u.seq * a.kv_heads + head) * a.cache_head;

  struct Tile {
    uint32_t k[4][NM], ks[4];
    uint32_t v[2][NV], vs[2][2];
  };
  auto load = [&](int t, Tile &x) {
    const uint8_t *tp = base + (int64_t)t * qtile_bytes(D);
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const int key = 32 * (kb / 2) + 8 * (i / 4) + 4 * (kb % 2) + i % 4;
      const uint8_t *kp = tp + key * (D / 2) + g * (D / 8);
      if constexpr (D == 128) {
        const u32x4 w = *(gptr16)kp;
#pragma unroll
        for (int m = 0; m < 4; ++m) x.k[kb][m] = w[m];
      } else {
        const uint2 w = *(const uint2 *)kp;
        x.k[kb][0] = w.x;
        x.k[kb][1] = w.y;
      }
      x.ks[kb] = tp[qtile_k_scales(D) + key * NG + (D == 128 ? g : g / 2)];
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int grp = 4 * c + g;
      const uint8_t *vp = tp + qtile_v(D) + (grp * (D / 4) + i * (NV / 4)) * 16;
#pragma unroll
      for (int e = 0; e < NV / 4; ++e) {
        const u32x4 w = *(gptr16)(vp + 16 * e);
#pragma unroll
        for (int m = 0; m < 4; ++m) x.v[c][4 * e + m] = w[m];
      }
      const uint2 s = *(const uint2 *)(tp + qtile_v_scales(D) + (grp * NG + i * NV / kQGroup) * 8);
      x.vs[c][0] = s.x;
      x.vs[c][1] = s.y;
    }
  };

  f32x4 acc[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) acc[j] = f32x4{};
  float m_run = kMInit, l_run = 0.f;

  auto work = [&](int t, const Tile &x) {
    f32x4 s[4];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      s[kb] = f32x4{};
      const float scale = __uint_as_float(x.ks[kb] << 23);
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        const uint32_t w = x.k[kb][m];
        const u32x4 kf = {values2<0>(w, scale), values2<1>(w, scale), values2<2>(w, scale), values2<3>(w, scale)};
        s[kb] = mfma16(__builtin_bit_cast(bf16x8, kf), qf[m], s[kb]);
      }
    }
    if ((t + 1) * KT > lo_all) {
      const int rem = hi - t * KT;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (32 * (kb / 2) + 8 * g + 4 * (kb % 2) + r >= rem) s[kb][r] = -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = larger(mx, s[kb][r]);
    mx *= sl2;
    if (__any(mx > m_run + kRescale)) {
      mx = larger_xor32(larger_xor16(mx));
      const float m_new = larger(m_run, mx);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int j = 0; j < NV; ++j) acc[j] *= alpha;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      bf16x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = __builtin_amdgcn_exp2f(fmaf(s[2 * c + e / 4][e % 4], sl2, -m_run));
        p[e] = (__bf16)y;
        l_run += (float)p[e];
      }
      uint32_t s0 = x.vs[c][0], s1 = x.vs[c][1];
      // slots behind the end hold anything: their scale becomes the smallest, so that a
      // probability of 0 times their value is 0
      const int left = u.nk - t * KT - 8 * (4 * c + g);
      if (left < 8) {
        s0 = left >= 4 ? s0 : left <= 0 ? 0u : s0 & ((1u << (8 * left)) - 1u);
        s1 = left <= 4 ? 0u : s1 & ((1u << (8 * (left - 4))) - 1u);
      }
      const float sc[8] = {scale_of<0>(s0), scale_of<1>(s0), scale_of<2>(s0), scale_of<3>(s0),
                           scale_of<0>(s1), scale_of<1>(s1), scale_of<2>(s1), scale_of<3>(s1)};
      u32x4 vf[NV];
#pragma unroll
      for (int e = 0; e < NV / 4; ++e)
#pragma unroll
        for (int m = 0; m < 4; ++m) {          // tokens 2 m and 2 m + 1, 4 dims
          const uint32_t w = x.v[c][4 * e + m];
          const uint32_t x0 = values2<0>(w, sc[2 * m]), x1 = values2<1>(w, sc[2 * m]);
          const uint32_t y0 = values2<2>(w, sc[2 * m + 1]), y1 = values2<3>(w, sc[2 * m + 1]);
          vf[4 * e + 0][m] = __builtin_amdgcn_perm(y0, x0, 0x05040100u);
          vf[4 * e + 1][m] = __builtin_amdgcn_perm(y0, x0, 0x07060302u);
          vf[4 * e + 2][m] = __builtin_amdgcn_perm(y1, x1, 0x05040100u);
          vf[4 * e + 3][m] = __builtin_amdgcn_perm(y1, x1, 0x07060302u);
        }
#pragma unroll
      for (int j = 0; j < NV; ++j) acc[j] = mfma16(__builtin_bit_cast(bf16x8, vf[j]), p, acc[j]);
    }
  };
  {
    Tile x, y;
    int t = t0 + wave;
    if (t < t1) load(t, x);
    while (t < t1) {
      if (t + kWaves < t1) load(t + kWaves, y);
      work(t, x);
      t += kWaves;
      if (t >= t1) break;
      if (t + kWaves < t1) load(t + kWaves, x);
      work(t, y);
      t += kWaves;
    }
  }

  // this wave's result: row i, dims NV (4 g + r) + j
  l_run = sum_xor32(sum_xor16(l_run));
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < NV; ++j) sO[wave][i][NV * (4 * g + r) + j] = acc[j][r];
  if (g == 0) {
    sM[wave][i] = m_run;
    sL[wave][i] = l_run;
  }
  __syncthreads();
  constexpr int TR = 64 * kWaves / R, ND = D / TR;       // threads per row, dims of a thread
  const int row = tid / TR, dim = tid % TR * ND;
  float M = sM[0][row];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sM[w][row]);
  float l = 0.f, o[ND] = {};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float f = __builtin_amdgcn_exp2f(sM[w][row] - M);
    l += f * sL[w][row];
#pragma unroll
    for (int e = 0; e < ND; ++e) o[e] += f * sO[w][row][dim + e];
  }
  if (u.row0 + row >= u.rows) return;
  if (!share.cut) {
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    const int rq = (u.row0 + row) / a.group, rh = head * a.group + (u.row0 + row - rq * a.group);
    uint16_t *op = a.o + (u.q0 + rq) * a.o_token + rh * a.o_head + dim;
#pragma unroll
    for (int e = 0; e < ND; e += 4) {
      const bf16x2 x = {(__bf16)(o[e] * inv), (__bf16)(o[e + 1] * inv)};
      const bf16x2 y = {(__bf16)(o[e + 2] * inv), (__bf16)(o[e + 3] * inv)};
      uint2 w;
      w.x = __builtin_bit_cast(uint32_t, x);
      w.y = __builtin_bit_cast(uint32_t, y);
      *reinterpret_cast<uint2 *>(op + e) = w;
    }
  } else {
    float *pp = a.part + share.slot * seq_part_floats(R, D);
#pragma unroll
    for (int e = 0; e < ND; e += 4)
      *reinterpret_cast<f32x4 *>(pp + row * D + dim + e) = f32x4{o[e], o[e + 1], o[e + 2], o[e + 3]};
    if (dim == 0) {
      pp[R * D + row] = M;
      pp[R * D + R + row] = l;
    }
  }
}

}  // namespace

hipError_t launch_decode(const SeqArgs &a, int head_dim, hipStream_t s) {
  const dim3 grid((uint32_t)seq_groups(a)), block(64 * kWaves);
  if (head_dim == 128) hipLaunchKernelGGL((decode_attn_kernel<128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((decode_attn_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace hc
