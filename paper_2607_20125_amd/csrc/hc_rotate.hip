// Rotary positions over several axes (time, height, width).
#include "hc_rotate.h"

#include <algorithm>

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// y = R(angle) x on pairs of dims, angle = position * theta^(-2 j / m).
//
// Bound by memory: each value is read and written once.  A thread owns 8 dims of a
// token (16 with the pairs half a head apart: both ends of its 8 pairs) in several
// heads, so that an angle is computed once and used by all of them, and 16 lanes
// read a 128-dim head's 256 bytes.  Angles: the position times the pair's turns per
// step in 64 bits, less the whole turns, then the hardware's sine and cosine of a
// fraction of a turn (8.5e-8 off at most over [-0.6, 0.6], measured).  No table: at
// 128 dims a token costs 64 sines and cosines against 3 KB and more of queries and keys.
// Measured: queries and keys of a 720P block (12 + 12 heads, 133 MB in and out) 21.6 to 27 us, 4.9 to
// 6.2 TB/s (more where the last outputs are still cached); 4099 tokens of 20 heads in float32 (84 MB) 17.5 us.
// ---------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kInFlight = 4;      // heads that a thread loads before it stores the first

template <typename XT, typename OT, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a) {
  constexpr int NP = HALVES ? 8 : 4;         // pairs of a thread
  constexpr int NV = HALVES ? 2 : 1;         // runs of 8 dims of a thread
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t token = at / a.items;
  const int item = (int)(at - token * a.items);
  if (token >= a.n_tokens) return;

  // the dims of this thread, and whether they turn
  const bool turning = item < (HALVES ? a.rot / 16 : a.rot / 8);
  int dim[NV];
  dim[0] = HALVES && !turning ? a.rot / 2 + 8 * item : 8 * item;
  if constexpr (HALVES) dim[1] = 8 * item + a.rot / 2;
  const bool second = HALVES && turning;

  float sn[NP], cs[NP];
  if (turning) turn_pairs<NP>(a, token, NP * item, sn, cs);

  const int h0 = blockIdx.y * a.heads_per, h1 = min(a.heads, h0 + a.heads_per);
  for (int h = h0; h < h1; h += kInFlight) {
    float x[kInFlight][NV][8];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (h + i >= h1) break;
      const bool two = h + i >= a.t[0].n_heads;
      const hc_rotate_tensor &t = a.t[two];
      const int64_t from = token * t.x_token + (int64_t)(h + i - (two ? a.t[0].n_heads : 0)) * t.x_head;
      load8<XT>(t.x, from + dim[0], x[i][0]);
      if constexpr (HALVES)
        if (second) load8<XT>(t.x, from + dim[1], x[i][1]);
    }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (h + i >= h1) break;
      if (turning) {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
          float &u = HALVES ? x[i][0][j] : x[i][0][2 * j];
          float &w = HALVES ? x[i][NV - 1][j] : x[i][0][2 * j + 1];
          const float y = u * cs[j] - w * sn[j];
          w = u * sn[j] + w * cs[j];
          u = y;
        }
      }
      const bool two = h + i >= a.t[0].n_heads;
      const hc_rotate_tensor &t = a.t[two];
      const int64_t to = token * t.out_token + (int64_t)(h + i - (two ? a.t[0].n_heads : 0)) * t.out_head;
      store8<OT>(t.out, to + dim[0], x[i][0]);
      if constexpr (HALVES)
        if (second) store8<OT>(t.out, to + dim[1], x[i][1]);
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &args, int x_type, int out_type, bool halves, hipStream_t s) {
  RotateArgs a = args;
  // threads per token: pairs of runs of 8 dims where they turn with the pairs half a head
  // apart, single runs elsewhere
  a.items = halves ? a.rot / 16 + (a.head_dim - a.rot) / 8 : a.head_dim / 8;
  const int64_t blocks = ((int64_t)a.n_tokens * a.items + kThreads - 1) / kThreads;
  // heads per thread: as many as leave 2048 work groups (8 for each CU), so that angles are
  // shared where there is work enough and few tokens still fill the card
  const int64_t cuts = std::min<int64_t>(a.heads, std::max<int64_t>(1, 2048 / std::max<int64_t>(1, blocks)));
  a.heads_per = (int)((a.heads + cuts - 1) / cuts);
  const dim3 grid((uint32_t)blocks, (uint32_t)((a.heads + a.heads_per - 1) / a.heads_per));
#define HC_ROT(X, O, H) hipLaunchKernelGGL((rotate_kernel<X, O, H>), grid, dim3(kThreads), 0, s, a)
#define HC_ROT_H(X, O) if (halves) HC_ROT(X, O, true); else HC_ROT(X, O, false)
  if (x_type == HC_BF16 && out_type == HC_BF16) { HC_ROT_H(uint16_t, uint16_t); }
  else if (x_type == HC_BF16) { HC_ROT_H(uint16_t, float); }
  else if (out_type == HC_BF16) { HC_ROT_H(float, uint16_t); }
  else { HC_ROT_H(float, float); }
#undef HC_ROT_H
#undef HC_ROT
  return hipGetLastError();
}

}  // namespace hc
