// Root-mean-square norm of every head, then rotary positions, in one pass; and the gradients.
#include "hc_rotate.h"
#include "hc_window.h"

namespace hc {
namespace {
using namespace dev;

// ---------------------------------------------------------------------------
// y = R(angle) (x r w),  r = (mean over the head's dims of x^2 + eps)^(-1/2).
//
// Bound by memory, as the rotation alone: each value is read and written once.  A thread owns
// 8 dims of a token (or both ends of 8 pairs half a head apart) in several heads, so that an angle is
// computed once; the 8, 16 or 32 lanes of a head add their squares up in the vector unit (lanes are
// mirrored and swapped in place: no LDS).  Sums, the norm and the rotation are in 32 bits, rounded once
// at the end.  A thread has 4 heads' loads in flight.  Queries and keys of a 720P block (10800 tokens, 12 + 12 heads of 128
// dims, bf16): 24 us, 5.4 TB/s, the rotation alone 23.
// ---------------------------------------------------------------------------
constexpr int kThreads = kNormThreads, kInFlight = kNormInFlight;

template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false));
}
// Sum over 2^bits neighbouring lanes, in all of them.  (Behind each step the lanes that it joined
// hold the same, so a mirror reaches the other half as well as an exchange would.)
__device__ __forceinline__ float sum_lanes(float x, int bits) {
  if (bits > 0) x = add_dpp<0xB1>(x);        // 1 0 3 2
  if (bits > 1) x = add_dpp<0x4E>(x);        // 2 3 0 1
  if (bits > 2) x = add_dpp<0x141>(x);       // mirrored in 8
  if (bits > 3) x = add_dpp<0x140>(x);       // mirrored in 16
  if (bits > 4) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// What a thread has of a head: NV runs of 8 dims, of which the second is there where pairs half a head
// apart turn.
template <bool HALVES>
struct Item {
  static constexpr int NP = HALVES ? 8 : 4, NV = HALVES ? 2 : 1;
  bool live, turning, second;
  int dim[2];
  __device__ __forceinline__ Item(const RotateArgs &r, int item) {
    live = item < (HALVES ? r.rot / 16 + (r.head_dim - r.rot) / 8 : r.head_dim / 8);
    turning = item < (HALVES ? r.rot / 16 : r.rot / 8);
    dim[0] = HALVES && !turning ? r.rot / 2 + 8 * item : 8 * item;
    dim[1] = 8 * item + r.rot / 2;
    second = HALVES && turning;
  }
  template <typename T>
  __device__ __forceinline__ void load(const void *p, int64_t at, float (&x)[NV][8]) const {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if (v == 0 ? live : second) load8<T>(p, at + dim[v], x[v]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) x[v][e] = 0.f;
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(void *p, int64_t at, const float (&x)[NV][8]) const {
    if (live) store8<T>(p, at + dim[0], x[0]);
    if constexpr (HALVES)
      if (second) store8<T>(p, at + dim[1], x[1]);
  }
  __device__ __forceinline__ void weights(const NormArgs &a, const void *p, float (&w)[NV][8]) const {
    if (p && a.weight_type == HC_BF16) return load<uint16_t>(p, 0, w);
    if (p) return load<float>(p, 0, w);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[v][e] = 1.f;
  }
  __device__ __forceinline__ void turn(float (&x)[NV][8], const float (&sn)[NP], const float (&cs)[NP]) const {
    if (!turning) return;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      float &u = HALVES ? x[0][j] : x[0][2 * j];
      float &w = HALVES ? x[NV - 1][j] : x[0][2 * j + 1];
      const float y = u * cs[j] - w * sn[j];
      w = u * sn[j] + w * cs[j];
      u = y;
    }
  }
};

// This work group's tensor, and its share of the heads.
struct Share {
  int tensor, cut, h0, h1;
};
__device__ __forceinline__ Share share_of(const NormArgs &a) {
  Share s;
  s.tensor = (int)blockIdx.y >= a.t[0].cuts;
  s.cut = (int)blockIdx.y - (s.tensor ? a.t[0].cuts : 0);
  const NormTensor &t = a.t[s.tensor];
  s.h0 = (int)((int64_t)t.n_heads * s.cut / t.cuts);
  s.h1 = (int)((int64_t)t.n_heads * (s.cut + 1) / t.cuts);
  return s;
}

template <typename XT, typename OT, bool HALVES>
__global__ __launch_bounds__(kThreads) void norm_rotate_kernel(NormArgs a) {
  using I = Item<HALVES>;
  const RotateArgs &r = a.rotate;
  const int64_t token = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> a.lane_bits;
  if (token >= r.n_tokens) return;
  const int lane = threadIdx.x & ((1 << a.lane_bits) - 1);
  const I item(r, lane);
  const Share s = share_of(a);
  const NormTensor &t = a.t[s.tensor];
  float w[I::NV][8], sn[I::NP], cs[I::NP];
  item.weights(a, t.weight, w);
  if (item.turning) turn_pairs<I::NP>(r, token, I::NP * lane, sn, cs);
  const float per = 1.f / (float)r.head_dim;

  for (int h = s.h0; h < s.h1; h += kInFlight) {
    float x[kInFlight][I::NV][8];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (h + i >= s.h1) break;
      item.template load<XT>(t.x, token * t.x_token + (int64_t)(h + i) * t.x_head, x[i]);
    }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (h + i >= s.h1) break;
      float ss = 0.f;
#pragma unroll
      for (int v = 0; v < I::NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x[i][v][e], x[i][v][e], ss);
      const float rms = __builtin_amdgcn_rsqf(fmaf(sum_lanes(ss, a.lane_bits), per, a.eps));
#pragma unroll
      for (int v = 0; v < I::NV; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][v][e] *= rms * w[v][e];
      item.turn(x[i], sn, cs);
      item.template store<OT>(t.y, token * t.y_token + (int64_t)(h + i) * t.y_head, x[i]);
    }
  }
}

// ---------------------------------------------------------------------------
// With n = x r, g' = R(-angle) dy and g = g' w:  dx = r (g - n mean(g n)),  dw = sum over tokens and
// heads of g' n.
//
// Bound by memory: x and dy in, dx out.  Threads own what they own in the forward pass and walk the tokens
// by the launch's work groups, adding dw up in registers; a work group's sums, joined in LDS, go to one row of the
// workspace, and a second launch adds those rows up in a fixed order, so that results repeat bit for bit.  Two heads in
// flight, or one with pairs half a head apart.  A 480P block (4680 tokens, 12 + 12 heads of 128 dims, bf16): 22 us, 3.9
// TB/s, and 4 for the second launch; 4099 tokens of 16 + 4 heads in 32 bits, positions given, 28 us, 4.5 TB/s, and 4.
// ---------------------------------------------------------------------------

template <typename XT, typename OT, bool HALVES>
__global__ __launch_bounds__(kThreads) void norm_rotate_backward_kernel(NormArgs a) {
  using I = Item<HALVES>;
  constexpr int kBackInFlight = HALVES ? 1 : 2;       // heads (with both ends of 8 pairs, two cost half of the waves)
  __shared__ float sw[kThreads * I::NV * 8];
  const RotateArgs &r = a.rotate;
  const int per_group = kThreads >> a.lane_bits, slot = threadIdx.x >> a.lane_bits;
  const int lane = threadIdx.x & ((1 << a.lane_bits) - 1);
  const I item(r, lane);
  const Share s = share_of(a);
  const NormTensor &t = a.t[s.tensor];
  float w[I::NV][8], dw[I::NV][8];
  item.weights(a, t.weight, w);
#pragma unroll
  for (int v = 0; v < I::NV; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[v][e] = 0.f;
  const float per = 1.f / (float)r.head_dim;

  for (int64_t token = (int64_t)blockIdx.x * per_group + slot; token < r.n_tokens; token += (int64_t)a.groups * per_group) {
    float sn[I::NP], cs[I::NP];
    if (item.turning) turn_pairs<I::NP>(r, token, I::NP * lane, sn, cs);
#pragma unroll
    for (int j = 0; j < I::NP; ++j) sn[j] = -sn[j];
    for (int h = s.h0; h < s.h1; h += kBackInFlight) {
      float x[kBackInFlight][I::NV][8], g[kBackInFlight][I::NV][8];
#pragma unroll
      for (int i = 0; i < kBackInFlight; ++i) {
        if (h + i >= s.h1) break;
        item.template load<XT>(t.x, token * t.x_token + (int64_t)(h + i) * t.x_head, x[i]);
        item.template load<OT>(t.y, token * t.y_token + (int64_t)(h + i) * t.y_head, g[i]);
      }
#pragma unroll
      for (int i = 0; i < kBackInFlight; ++i) {
        if (h + i >= s.h1) break;
        item.turn(g[i], sn, cs);
        float ss = 0.f, gx = 0.f;
#pragma unroll
        for (int v = 0; v < I::NV; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss = fmaf(x[i][v][e], x[i][v][e], ss);
            gx = fmaf(g[i][v][e] * w[v][e], x[i][v][e], gx);
          }
        const float rms = __builtin_amdgcn_rsqf(fmaf(sum_lanes(ss, a.lane_bits), per, a.eps));
        const float mean = sum_lanes(gx, a.lane_bits) * rms * per;      // of g n
#pragma unroll
        for (int v = 0; v < I::NV; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float n = x[i][v][e] * rms;
            dw[v][e] = fmaf(g[i][v][e], n, dw[v][e]);
            x[i][v][e] = rms * fmaf(-n, mean, g[i][v][e] * w[v][e]);
          }
        item.template store<XT>(t.dx, token * t.dx_token + (int64_t)(h + i) * t.dx_head, x[i]);
      }
    }
  }
  if (!t.dweight) return;
  // slot by slot, in order
#pragma unroll
  for (int v = 0; v < I::NV; ++v)
    if (v == 0 ? item.live : item.second)
#pragma unroll
      for (int e = 0; e < 8; ++e) sw[slot * r.head_dim + item.dim[v] + e] = dw[v][e];
  __syncthreads();
  if ((int)threadIdx.x >= r.head_dim) return;
  float sum = 0.f;
  for (int i = 0; i < per_group; ++i) sum += sw[i * r.head_dim + threadIdx.x];
  const int64_t first = s.tensor ? norm_parts(a, 0) : 0;
  a.part[(first + (int64_t)s.cut * a.groups + blockIdx.x) * r.head_dim + threadIdx.x] = sum;
}

// dw of 8 dims of a tensor: 128 threads a dim add every 128th row, and are joined in LDS, 16 and then 8 of them.  (With 32 threads a
// dim: a 480P block's gradients from memory 33.4 us instead of 31.6.)
constexpr int kWeightThreads = 1024;
__global__ __launch_bounds__(kWeightThreads) void norm_weights_kernel(NormArgs a) {
  constexpr int each = kWeightThreads / 8;
  __shared__ float sw[kWeightThreads], half[64];
  const NormTensor &t = a.t[blockIdx.y];
  if (!t.dweight) return;
  const int d = threadIdx.x % 8, first = threadIdx.x / 8, dim = blockIdx.x * 8 + d;
  const int64_t rows = norm_parts(a, blockIdx.y);
  const float *p = a.part + (blockIdx.y ? norm_parts(a, 0) : 0) * a.rotate.head_dim + dim;
  float sum = 0.f;
#pragma unroll 8
  for (int64_t i = first; i < rows; i += each) sum += p[i * a.rotate.head_dim];
  sw[threadIdx.x] = sum;
  __syncthreads();
  if (first < 8) {
    sum = 0.f;
    for (int i = 0; i < each / 8; ++i) sum += sw[(first * (each / 8) + i) * 8 + d];
    half[threadIdx.x] = sum;
  }
  __syncthreads();
  if (first) return;
  for (int i = 1; i < 8; ++i) sum += half[i * 8 + d];
  t.dweight[dim] = sum;
}

}  // namespace

#define HC_NORM_TYPES(K, ...)                                                        \
  if (x_type == HC_BF16 && out_type == HC_BF16) { HC_NORM_HALVES(K, uint16_t, uint16_t); } \
  else if (x_type == HC_BF16) { HC_NORM_HALVES(K, uint16_t, float); }                \
  else if (out_type == HC_BF16) { HC_NORM_HALVES(K, float, uint16_t); }              \
  else { HC_NORM_HALVES(K, float, float); }
#define HC_NORM_HALVES(K, X, O)                                                      \
  if (halves) hipLaunchKernelGGL((K<X, O, true>), grid, dim3(kThreads), 0, s, a);    \
  else hipLaunchKernelGGL((K<X, O, false>), grid, dim3(kThreads), 0, s, a)

hipError_t launch_norm(const NormArgs &a, int x_type, int out_type, bool halves, hipStream_t s) {
  const dim3 grid((uint32_t)a.groups, (uint32_t)(a.t[0].cuts + (a.n_tensors > 1 ? a.t[1].cuts : 0)));
  HC_NORM_TYPES(norm_rotate_kernel)
  return hipGetLastError();
}

hipError_t launch_norm_backward(const NormArgs &a, int x_type, int out_type, bool halves, hipStream_t s) {
  const dim3 grid((uint32_t)a.groups, (uint32_t)(a.t[0].cuts + (a.n_tensors > 1 ? a.t[1].cuts : 0)));
  if (a.groups > 0) { HC_NORM_TYPES(norm_rotate_backward_kernel) }
  const bool weights = a.t[0].dweight || (a.n_tensors > 1 && a.t[1].dweight);
  if (weights)
    hipLaunchKernelGGL(norm_weights_kernel, dim3((uint32_t)(a.rotate.head_dim / 8), (uint32_t)a.n_tensors), dim3(kWeightThreads), 0, s, a);
  return hipGetLastError();
}
#undef HC_NORM_HALVES
#undef HC_NORM_TYPES

}  // namespace hc
