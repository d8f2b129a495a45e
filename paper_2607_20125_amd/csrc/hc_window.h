// Internal structures of the operators of a model with a sliding window (hc_window.cpp, hc_norm.hip,
// hc_paged.hip, hc_window_grad.h, and the kernels of hc_seq.hip and hc_seq128.hip).  Not part of the public ABI.
#pragma once

#include "hc_ops.h"

namespace hc {

// --- norm and rotary positions ----------------------------------------------------
struct NormTensor {
  const void *x, *weight;        // weight may be null: ones
  void *y;                       // forward: the output; backward: the output's gradient, which is read
  void *dx;                      // backward
  float *dweight;                // backward, may be null
  int64_t x_token, x_head, y_token, y_head, dx_token, dx_head;
  int32_t n_heads, cuts;         // work groups that share the heads of a token
};
struct NormArgs {
  RotateArgs rotate;             // its tensors are not used
  NormTensor t[2];
  int32_t n_tensors, weight_type;
  int32_t lane_bits;             // 2^lane_bits lanes take a token's head
  int32_t groups;                // work groups along the tokens
  float eps;
  float *part;                   // backward: [tensor][work group][head_dim] sums of the weights' gradients
};
constexpr int kNormThreads = 256;
constexpr int kNormInFlight = 4;   // heads that a thread loads before it uses the first
// Lanes that a token's head needs.
inline int norm_items(const RotateArgs &r, bool halves) { return halves ? r.rot / 16 + (r.head_dim - r.rot) / 8 : r.head_dim / 8; }
// Partial sums of the weights' gradients of tensor i, and where they begin.
inline __host__ __device__ int64_t norm_parts(const NormArgs &a, int i) { return (int64_t)a.groups * a.t[i].cuts; }
hipError_t launch_norm(const NormArgs &a, int x_type, int out_type, bool halves, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs &a, int x_type, int out_type, bool halves, hipStream_t s);

// --- pages ----------------------------------------------------------------------------
struct PagedRowsArgs {
  hc_pages pages;
  hc_page_table table;
  hc_qcache_rows rows;
  int32_t page_shift;
};
hipError_t launch_paged_append(const PagedRowsArgs &a, hipStream_t s);

// --- attention with a window ------------------------------------------------------------
// By waves of 32 rows (hc_seq.hip) or of 64 (hc_seq128.hip), and for few rows (hc_paged.hip).
hipError_t launch_window(const SeqArgs &a, int head_dim, hipStream_t s);
hipError_t launch_window128(const SeqArgs &a, hipStream_t s);
hipError_t launch_paged_decode(const SeqArgs &a, int head_dim, hipStream_t s);

// Gradients.  Rows and units are those of the forward pass; key units are runs of kGradKeys keys of a sequence.
constexpr int kGradKeys = 128;
struct GradArgs {
  SeqArgs seq;                   // q, k, v, the mask; o is the forward output, which is read
  const uint16_t *dout;
  const float *lse;              // [heads][n_tokens]
  uint16_t *dq, *dk, *dv;
  int64_t do_token, do_head, dq_token, dq_head, dk_token, dk_head, dv_token, dv_head;
  float *stats;                  // [2][heads][n_tokens]: -lse / scale, -(sum over dims of dout * o)
  int32_t key_tiles;             // key units that the launch has room for
  float scale;
  // key units are cut into pieces of rows, whose partial gradients a further launch adds up in order
  int32_t n_split;
  float *part;                   // [key unit][kv head][n_split][2][kGradKeys][d]
};
hipError_t launch_grad64(const GradArgs &a, hipStream_t s);
hipError_t launch_grad128(const GradArgs &a, hipStream_t s);

}  // namespace hc
