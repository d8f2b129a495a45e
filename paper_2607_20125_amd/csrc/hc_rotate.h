// Device-side pieces of the rotation, alone (hc_rotate.hip) and behind a norm (hc_norm.hip).
// Included by the .hip sources only.
#pragma once

#include "hc_device.h"
#include "hc_ops.h"

namespace hc {
namespace dev {

// 8 neighbouring dims as floats, and back, rounded once.
template <typename T>
__device__ __forceinline__ void load8(const void *p, int64_t at, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4 w = gld16((const uint16_t *)p + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    const u32x4 a = gld16((const uint16_t *)((const float *)p + at));
    const u32x4 b = gld16((const uint16_t *)((const float *)p + at + 4));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __uint_as_float(a[i]);
      x[4 + i] = __uint_as_float(b[i]);
    }
  }
}

template <typename T>
__device__ __forceinline__ void store8(void *p, int64_t at, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 r = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
      w[i] = __builtin_bit_cast(uint32_t, r);
    }
    *reinterpret_cast<u32x4 *>((uint16_t *)p + at) = w;
  } else {
    float *o = (float *)p + at;
    *reinterpret_cast<f32x4 *>(o) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(o + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// Sines (with the rotation's sign) and cosines of pairs first .. first + NP - 1 of a token.
template <int NP>
__device__ __forceinline__ void turn_pairs(const RotateArgs &a, int64_t token, int first, float (&sn)[NP], float (&cs)[NP]) {
  int pos[kRotMaxAxes];
  if (a.positions) {
#pragma unroll
    for (int i = 0; i < kRotMaxAxes; ++i)
      if (i < a.n_axes) pos[i] = a.positions[(int64_t)i * a.n_tokens + token];
  } else {
    const uint32_t t = (uint32_t)token, row = t / (uint32_t)a.grid_w;
    const uint32_t frame = row / (uint32_t)a.grid_h;
    pos[0] = a.frame0 + (int)frame;
    pos[1] = (int)(row - frame * a.grid_h);
    pos[2] = (int)(t - row * a.grid_w);
  }
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int pair = first + j;
    int p = pos[0];
#pragma unroll
    for (int i = 1; i < kRotMaxAxes; ++i)
      if (i < a.n_axes && pair >= a.axis_end[i - 1]) p = pos[i];
    const double turns = (double)p * a.turns[pair];
    const float part = (float)(turns - __builtin_rint(turns));
    cs[j] = __builtin_amdgcn_cosf(part);
    sn[j] = __builtin_amdgcn_sinf(part) * a.sign;
  }
}

}  // namespace dev
}  // namespace hc
