// The cache in pages: storing rows, and its attention for few rows per sequence (single tokens).
#include "hc_mask.h"
#include "hc_window.h"

#include <algorithm>

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// Append: a work group takes 4 tokens and a share of their heads.  Each wave finds the place of one token
// (its lanes search the offsets 64 at a time), then all threads copy 16-byte pieces of keys and values.
// Bound by memory: 2 bytes in and 2 out a value; with few tokens by the chain offsets, start, table.  A 480P block of 12 heads of
// 128 dims 11 us, 5.2 TB/s; one token of each of 64 sequences, 8 heads, 3 us.
// ---------------------------------------------------------------------------
constexpr int kAppendThreads = 256, kAppendTokens = 4;

// The last sequence that starts at or before `row` (empty ones start there too), by a whole wave.
__device__ __forceinline__ int find_sequence(const int32_t *cu, int n_seqs, int row, int lane) {
  int low = 0, len = n_seqs;
  while (len > 1) {
    const int step = (len + 63) / 64, at = low + lane * step;
    const uint64_t before = __ballot(lane * step < len && cu[min(at, n_seqs)] <= row);
    const int k = max((int)__popcll(before) - 1, 0);
    len = min(step, len - k * step);
    low += k * step;
  }
  return low;
}

template <int D>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(PagedRowsArgs a) {
  constexpr int C = D / 8;       // 16-byte pieces of a head
  __shared__ int64_t sPage[kAppendTokens];
  __shared__ int sToken[kAppendTokens];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * kAppendTokens;
  {
    const int64_t row = row0 + wave;
    int64_t page = -1;
    int64_t slot = 0;
    if (row < a.rows.n_tokens) {
      int seq;
      int64_t in_seq;
      bool ok = true;
      if (a.rows.cu_seqlens) {
        seq = find_sequence(a.rows.cu_seqlens, a.table.n_seqs, (int)row, lane);
        in_seq = row - a.rows.cu_seqlens[seq];
        ok = in_seq >= 0 && row < a.rows.cu_seqlens[seq + 1];
      } else {
        const int per = a.rows.n_tokens / a.table.n_seqs;
        seq = (int)(row / per);
        in_seq = row - (int64_t)seq * per;
      }
      slot = in_seq + a.rows.start[seq];
      if (ok && slot >= 0 && slot >> a.page_shift < a.table.max_pages) {
        page = a.table.table[seq * a.table.stride + (slot >> a.page_shift)];
        if (page >= a.pages.n_pages) page = -1;
      }
    }
    if (lane == 0) {
      sPage[wave] = page;
      sToken[wave] = (int)(slot & ((1 << a.page_shift) - 1));
    }
  }
  __syncthreads();
  const int H = a.pages.n_heads;
  const int h0 = (int)((int64_t)H * blockIdx.y / gridDim.y), nh = (int)((int64_t)H * (blockIdx.y + 1) / gridDim.y) - h0;
  for (int i = threadIdx.x; i < kAppendTokens * nh * C; i += kAppendThreads) {
    const int c = i % C, r = i / C % kAppendTokens, h = h0 + i / C / kAppendTokens;
    const int64_t page = sPage[r], token = sToken[r];
    if (page < 0) continue;
    const u32x4 k = gld16((const uint16_t *)a.rows.k + (row0 + r) * a.rows.k_token + h * a.rows.k_head + c * 8);
    const u32x4 v = gld16((const uint16_t *)a.rows.v + (row0 + r) * a.rows.v_token + h * a.rows.v_head + c * 8);
    *(u32x4 *)((uint16_t *)a.pages.k + page * a.pages.k_page + token * a.pages.k_token + h * a.pages.k_head + c * 8) = k;
    *(u32x4 *)((uint16_t *)a.pages.v + page * a.pages.v_page + token * a.pages.v_token + h * a.pages.v_head + c * 8) = v;
  }
}

// ---------------------------------------------------------------------------
// One work group: up to 16 rows (queries times query heads of one key head) of a sequence over one
// range of its key tiles; its 4 waves take every fourth tile and are merged in LDS at the end.
//
// Bound by the cache's bytes.  Nothing is shared between waves, so keys and values go from memory to
// registers, half a tile (32 keys) ahead, and are operands of the matrix cores without passing LDS:
//  * S^T = K Q^T with 16x16x32 products: a lane's 16 bytes are 8 dims of one key.  Key rows are
//    fed so that lane group g ends up with keys 8 g .. 8 g + 7 of the 32.
//  * O^T = V^T P^T needs 8 keys of one dim: a lane loads D / 16 dims of 8 keys and transposes them in
//    registers, two keys of a dim by one byte permute.  The probabilities are rounded to bf16 for it, and their sum
//    is of the rounded ones (see hc_seq.hip).
// The pages of a tile are looked up a tile ahead.  One token of 32 heads over 131072 keys of 8 heads of 128 dims in pages of 64:
// 95 us, 5.6 TB/s, and 5 for the merge; a token each of 48 sequences of up to 8192 keys, window 2048, 7 x 4 heads of
// 64 dims, pages of 16: 21 us, 4.2 TB/s, and 4.5.
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
__global__ __launch_bounds__(64 * kWaves, 2) void paged_decode_kernel(SeqArgs a) {
  constexpr int R = kDecodeRows, KT = kSeqKeys;
  constexpr int NM = D / 32;             // score products per 16 keys
  constexpr int NV = D / 16;             // output products per 32 keys; dims of a lane's V piece
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
    const uint16_t *qp = a.q + (u.q0 + qi) * a.q_token + qh * a.q_head + 8 * g;
#pragma unroll
    for (int m = 0; m < NM; ++m) qf[m] = ld_g16(qp + 32 * m);
  }
  const Seen mine = seen_by(a, u, qi);
  const int last = min(u.row0 + R, u.rows) - 1;
  const KeyTiles tiles(seen_by(a, u, u.row0 / a.group), seen_by(a, u, last / a.group));
  int t0, t1;
  key_range(a, u, share, tiles.n, t0, t1);
  const float sl2 = a.scale_log2;

  struct Half {
    u32x4 k[2][NM];
    uint32_t v[8][NV / 2];
  };
  const uint16_t *kh = a.k + head * a.k_head + 8 * g, *vh = a.v + head * a.v_head + NV * i;
  // half c of the tile at this place, whose runs' table entries are `entries`
  auto load = [&](int place, int c, int entries, Half &x) {
    auto base = [&](const uint16_t *p, int64_t page, int64_t token, int j) {
      return p + page_of(a, entries, j) * page + run_token(a, run_of(u, place, j)) * token;
    };
    const int r0 = run_of(u, place, 2 * c) * 16, r1 = run_of(u, place, 2 * c + 1) * 16;
    {
      const uint16_t *p0 = base(kh, a.k_page, a.k_token, 2 * c), *p1 = base(kh, a.k_page, a.k_token, 2 * c + 1);
      const uint16_t *p = i >= 8 ? p1 : p0;
      const int r = i >= 8 ? r1 : r0;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int key = place * KT + 32 * c + 8 * (i / 4) + 4 * kb + i % 4;
        const uint16_t *q = p + (min(key, u.nk - 1) - r) * a.k_token;
#pragma unroll
        for (int m = 0; m < NM; ++m) x.k[kb][m] = gld16(q + 32 * m);
      }
    }
    const uint16_t *p0 = base(vh, a.v_page, a.v_token, 2 * c), *p1 = base(vh, a.v_page, a.v_token, 2 * c + 1);
    const uint16_t *p = g >= 2 ? p1 : p0;
    const int r = g >= 2 ? r1 : r0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint16_t *q = p + (min(place * KT + 32 * c + 8 * g + e, u.nk - 1) - r) * a.v_token;
      if constexpr (D == 128) {
        const u32x4 w = gld16(q);
#pragma unroll
        for (int m = 0; m < 4; ++m) x.v[e][m] = w[m];
      } else {
        const uint2 w = *(const uint2 *)q;
        x.v[e][0] = w.x;
        x.v[e][1] = w.y;
      }
    }
  };

  f32x4 acc[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) acc[j] = f32x4{};
  float m_run = kMInit, l_run = 0.f;

  auto work = [&](int place, int c, uint32_t absent, Half &x) {
    f32x4 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      s[kb] = f32x4{};
#pragma unroll
      for (int m = 0; m < NM; ++m) s[kb] = mfma16(__builtin_bit_cast(bf16x8, x.k[kb][m]), qf[m], s[kb]);
    }
    if (!tiles.whole(place, a.sinks) || absent) {
      const bool gone = absent >> (2 * c + (g >> 1)) & 1;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (gone | !mine.sees(place * KT + 32 * c + 8 * g + 4 * kb + r)) s[kb][r] = -INFINITY;
      if (gone)                // any values may stand there: a probability of 0 times 0 is 0
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int m = 0; m < NV / 2; ++m) x.v[e][m] = 0;
    }
    float mx = s[0][0];
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = larger(mx, larger(s[0][r], s[1][r]));
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
    bf16x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = (__bf16)__builtin_amdgcn_exp2f(fmaf(s[e / 4][e % 4], sl2, -m_run));
      l_run += (float)p[e];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      u32x4 vf;
#pragma unroll
      for (int m = 0; m < 4; ++m)
        vf[m] = __builtin_amdgcn_perm(x.v[2 * m + 1][j / 2], x.v[2 * m][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
      acc[j] = mfma16(__builtin_bit_cast(bf16x8, vf), p, acc[j]);
    }
  };
  {
    Half x, y;
    int t = t0 + wave;
    int entries = 0;
    if (t < t1) {
      entries = page_entry(a, u, tiles.place(t), lane);
      load(tiles.place(t), 0, entries, x);
    }
    for (; t < t1; t += kWaves) {
      const int place = tiles.place(t), next = tiles.place(t + kWaves);
      const uint32_t absent = absent_runs(a, entries);
      const int entries_next = page_entry(a, u, next, lane);
      load(place, 1, entries, y);
      work(place, 0, absent, x);
      if (t + kWaves < t1) load(next, 0, entries_next, x);
      work(place, 1, absent, y);
      entries = entries_next;
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

hipError_t launch_paged_append(const PagedRowsArgs &a, hipStream_t s) {
  const int64_t groups = ((int64_t)a.rows.n_tokens + kAppendTokens - 1) / kAppendTokens;
  // heads are shared out until 1024 work groups run
  const int64_t shares = std::min<int64_t>(a.pages.n_heads, std::max<int64_t>(1, 1024 / groups));
  const dim3 grid((uint32_t)groups, (uint32_t)shares), block(kAppendThreads);
  if (a.pages.head_dim == 128) hipLaunchKernelGGL(paged_append_kernel<128>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(paged_append_kernel<64>, grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_decode(const SeqArgs &a, int head_dim, hipStream_t s) {
  const dim3 grid((uint32_t)seq_groups(a)), block(64 * kWaves);
  if (head_dim == 128) hipLaunchKernelGGL((paged_decode_kernel<128>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((paged_decode_kernel<64>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace hc
