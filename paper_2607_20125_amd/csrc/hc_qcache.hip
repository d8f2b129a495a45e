// The 4-bit key/value cache: storing rows and reading them back.
#include "hc_device.h"
#include "hc_seq.h"

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// Append: a thread takes 32 dims of one token, head and tensor, the values that
// share a scale.  Consecutive lanes take 8 tokens, then the 32-dim groups of a head: the
// codes of a V group of 8 tokens are interleaved by token.
//
// Bound by memory: append reads 2 bytes a value and writes 17/32, read the reverse (84 MB each
// for a 720P block of 12 heads: 20.9 us and 23.4 us, 4.0 and 3.6 TB/s).
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;

struct Place {
  bool ok;
  int64_t row;             // of k and v
  int head, grp;           // 32-dim group
  bool is_v;
  uint8_t *tile;           // of the cache
  int at;                  // token of the tile
};

template <int D>
__device__ __forceinline__ Place place(const QCacheArgs &a, int64_t i, int low) {
  constexpr int NG = D / kQGroup;
  Place p;
  const int H = a.cache.n_heads;
  p.grp = (int)(i % NG);
  i /= NG;
  p.head = (int)(i % H);
  i /= H;
  p.is_v = i & 1;
  p.row = (i >> 1) * 8 + low;
  p.ok = p.row < a.rows.n_tokens;
  p.tile = nullptr;
  p.at = 0;
  if (!p.ok) return p;
  int seq;
  int64_t in_seq;
  if (a.rows.cu_seqlens) {
    // the last sequence that starts at or before the row (empty ones start there too)
    int lo = 0, hi = a.cache.n_seqs;
    while (lo + 1 < hi) {
      const int mid = (lo + hi) / 2;
      if (a.rows.cu_seqlens[mid] <= p.row) lo = mid;
      else hi = mid;
    }
    seq = lo;
    in_seq = p.row - a.rows.cu_seqlens[seq];
    p.ok = in_seq >= 0 && p.row < a.rows.cu_seqlens[seq + 1];
  } else {
    const int per = a.rows.n_tokens / a.cache.n_seqs;
    seq = (int)(p.row / per);
    in_seq = p.row - (int64_t)seq * per;
  }
  const int64_t slot = in_seq + a.rows.start[seq];
  p.ok = p.ok && slot >= 0 && slot < a.cache.capacity;
  if (!p.ok) return p;
  p.tile = (uint8_t *)a.cache.data + ((int64_t)seq * H + p.head) * qcache_head_bytes(a.cache.capacity, D) +
           slot / kQTokens * qtile_bytes(D);
  p.at = (int)(slot % kQTokens);
  return p;
}

// Bytes of the codes: K's 16 side by side, V's in 8 pieces of 2, 16 apart.
template <int D>
__device__ __forceinline__ uint8_t *codes_at(const Place &p) {
  return p.is_v ? p.tile + qtile_v(D) + ((p.at / 8) * (D / 4) + p.grp * 8) * 16 + (p.at % 8) * 2
                : p.tile + p.at * (D / 2) + p.grp * 16;
}
template <int D>
__device__ __forceinline__ uint8_t *scale_at(const Place &p) {
  return p.is_v ? p.tile + qtile_v_scales(D) + ((p.at / 8) * (D / kQGroup) + p.grp) * 8 + p.at % 8
                : p.tile + qtile_k_scales(D) + p.at * (D / kQGroup) + p.grp;
}

// Biased exponent of the scale for 32 values whose largest magnitude has these bits:
// the power of two of the magnitude, less 2, one more where its fraction exceeds
// 7/4 (which still rounds to 6 by half a step).
__device__ __forceinline__ uint32_t scale_code(uint32_t top) {
  if (top >= 0x7f800000u) return kScaleNone;
  const int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(e, kScaleLow), kScaleHigh);
}

// The 8x8 matrix of 2-byte elements that 8 neighbouring lanes hold (lane r: row r in four words)
// transposed (lane c: column c), in three exchanges with the lanes 4, 2 and 1 away: halves
// of 4, 2 and 1 elements change places.
__device__ __forceinline__ u32x4 transpose8(u32x4 w) {
  const int lane = threadIdx.x & 7;
  auto from = [](uint32_t x, int d) { return (uint32_t)__shfl_xor((int)x, d); };
  {
    const bool up = lane & 4;          // keeps words 2, 3 and gives away 0, 1
    const uint32_t g0 = from(up ? w[0] : w[2], 4), g1 = from(up ? w[1] : w[3], 4);
    w = up ? u32x4{g0, g1, w[2], w[3]} : u32x4{w[0], w[1], g0, g1};
  }
  {
    const bool up = lane & 2;
    const uint32_t g0 = from(up ? w[0] : w[1], 2), g1 = from(up ? w[2] : w[3], 2);
    w = up ? u32x4{g0, w[1], g1, w[3]} : u32x4{w[0], g0, w[2], g1};
  }
  const bool up = lane & 1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i], g = from(x, 1);
    // even lane: (x low, g low); odd lane: (g high, x high)
    w[i] = up ? __builtin_amdgcn_perm(x, g, 0x07060302u) : __builtin_amdgcn_perm(g, x, 0x05040100u);
  }
  return w;
}

// Whether the 8 lanes of a row of 8 hold the 8 tokens of one group of the cache's tiles: then their V
// codes make 8 whole pieces of 16 bytes, one for each lane after a transposition.
__device__ __forceinline__ bool whole_group(const Place &p) {
  const uint64_t good = __ballot(p.ok && p.at % 8 == (int)(threadIdx.x & 7));
  const int first = (threadIdx.x & 63) & ~7;
  // (lanes whose tokens are the right ones of different groups belong to different tiles or
  // sequences; then their row numbers do not continue their slots)
  const uint64_t base = (uint64_t)(uintptr_t)p.tile + (uint64_t)(p.at / 8);
  const uint32_t lo = (uint32_t)base, hi = (uint32_t)(base >> 32);
  const int src = first;
  const bool same = lo == (uint32_t)__shfl((int)lo, src) && hi == (uint32_t)__shfl((int)hi, src);
  const uint64_t alike = __ballot(same);
  return ((good & alike) >> first & 0xffu) == 0xffu;
}

template <int D>
__global__ __launch_bounds__(kThreads) void qcache_append_kernel(QCacheArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const Place p = place<D>(a, i >> 3, (int)(i & 7));
  u32x4 c = {0, 0, 0, 0};
  uint32_t code = 0;
  if (p.ok) {
    const uint16_t *src = p.is_v ? (const uint16_t *)a.rows.v + p.row * a.rows.v_token + p.head * a.rows.v_head
                                 : (const uint16_t *)a.rows.k + p.row * a.rows.k_token + p.head * a.rows.k_head;
    u32x4 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = gld16(src + p.grp * kQGroup + 8 * i);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        top = max(top, max(w[i][j] << 16 & 0x7fffffffu, w[i][j] & 0x7fff0000u));
    code = scale_code(top);
    // the conversion divides by the scale, rounds to even and saturates at 6
    const float scale = __uint_as_float(min(code, (uint32_t)kScaleHigh) << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w0 = w[i][0], w1 = w[i][1], w2 = w[i][2], w3 = w[i][3];
      uint32_t r = 0;
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w0), scale, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w1), scale, 1);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w2), scale, 2);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w3), scale, 3);
      c[i] = r;
    }
  }
  // (K and V alternate by runs of 8 lanes and more, so a run of 8 is of one kind)
  const bool whole = whole_group(p) && p.is_v;
  const u32x4 turned = transpose8(c);
  if (!p.ok) return;
  uint8_t *to = codes_at<D>(p);
  if (!p.is_v) {
    *(u32x4 *)to = c;
  } else if (whole) {
    // lane l has piece l (4 dims) of the 8 tokens; `to` is piece 0 of token l
    const int l = threadIdx.x & 7;
    *(u32x4 *)(to - 2 * l + 16 * l) = turned;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      *(uint16_t *)(to + 32 * i) = (uint16_t)c[i];
      *(uint16_t *)(to + 32 * i + 16) = (uint16_t)(c[i] >> 16);
    }
  }
  *scale_at<D>(p) = (uint8_t)code;
}

// A thread takes 8 dims of a token here, so that a row leaves in whole lines (32 dims a thread, 16 bytes
// of every 64 at a time: 27 us for the 66 MB of a 720P block).
template <int D>
__global__ __launch_bounds__(kThreads) void qcache_read_kernel(QCacheArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int c = (int)(i % (D / 8));          // 8-dim chunk of the head
  const int64_t j = i / (D / 8);
  const Place p = place<D>(a, (j >> 3) * (D / kQGroup) + c / 4, (int)(j & 7));
  if (!p.ok) return;
  const uint8_t *from = codes_at<D>(p);
  uint32_t w;
  if (p.is_v) {
    from += 32 * (c % 4);
    w = *(const uint16_t *)from | (uint32_t) * (const uint16_t *)(from + 16) << 16;
  } else {
    w = *(const uint32_t *)(from + 4 * (c % 4));
  }
  const float scale = __uint_as_float((uint32_t)*scale_at<D>(p) << 23);
  uint16_t *dst = p.is_v ? (uint16_t *)a.rows.v + p.row * a.rows.v_token + p.head * a.rows.v_head
                         : (uint16_t *)a.rows.k + p.row * a.rows.k_token + p.head * a.rows.k_head;
  *(u32x4 *)(dst + 8 * c) = u32x4{values2<0>(w, scale), values2<1>(w, scale), values2<2>(w, scale), values2<3>(w, scale)};
}

template <class F128, class F64>
hipError_t launch_rows(const QCacheArgs &a, int dims, F128 f128, F64 f64) {      // dims of a thread
  const int64_t threads = ((int64_t)a.rows.n_tokens + 7) / 8 * 8 * a.cache.n_heads * 2 * (a.cache.head_dim / dims);
  const uint32_t grid = (uint32_t)((threads + kThreads - 1) / kThreads);
  if (a.cache.head_dim == 128) f128(grid);
  else f64(grid);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qcache_append(const QCacheArgs &a, hipStream_t s) {
  return launch_rows(
      a, kQGroup, [&](uint32_t grid) { hipLaunchKernelGGL(qcache_append_kernel<128>, dim3(grid), dim3(kThreads), 0, s, a); },
      [&](uint32_t grid) { hipLaunchKernelGGL(qcache_append_kernel<64>, dim3(grid), dim3(kThreads), 0, s, a); });
}
hipError_t launch_qcache_read(const QCacheArgs &a, hipStream_t s) {
  return launch_rows(
      a, 8, [&](uint32_t grid) { hipLaunchKernelGGL(qcache_read_kernel<128>, dim3(grid), dim3(kThreads), 0, s, a); },
      [&](uint32_t grid) { hipLaunchKernelGGL(qcache_read_kernel<64>, dim3(grid), dim3(kThreads), 0, s, a); });
}

}  // namespace hc
