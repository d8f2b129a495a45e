// Checks of arguments and plans that the entry points of the operators beside the routed attention
// share (hc_ops.cpp, hc_window.cpp).
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "hc_context.h"
#include "hc_ops.h"

namespace hc {

// The context's device is current inside a call, the caller's again behind it.
struct OnDevice {
  int before = -1;
  hipError_t status;
  explicit OnDevice(int device) {
    status = hipGetDevice(&before);
    if (status == hipSuccess && before == device) before = -1;
    else if (status == hipSuccess) status = hipSetDevice(device);
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

constexpr float kLog2E = 1.4426950408889634f;

inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// Work groups of a launch dimension, of 256 threads at most: the runtime counts threads in 32 bits.
inline bool good_grid(int64_t groups) { return groups <= (int64_t)UINT32_MAX / 256; }

// A tensor of rows that are moved as 16-byte vectors.  (The stride of an axis of length 1 says nothing.)
struct Rows {
  const char *name;
  const void *p;
  int64_t token, head, n_tokens, n_heads;
};
inline hc_status check_tensor(hc_ctx *c, const Rows &t) {
  if (!t.p || !aligned16(t.p)) return fail(c, HC_E_INVAL, "%s must be a 16-byte aligned device pointer", t.name);
  auto good = [](int64_t stride, int64_t n) { return n <= 1 || (stride >= 0 && stride % 8 == 0); };
  if (!good(t.token, t.n_tokens) || !good(t.head, t.n_heads))
    return fail(c, HC_E_INVAL, "%s: strides must be multiples of 8 and not negative", t.name);
  return HC_OK;
}

// A tensor that a call writes: besides, no two of its rows of `dim` values overlap.
inline hc_status check_output(hc_ctx *c, const Rows &t, int dim) {
  hc_status st = check_tensor(c, t);
  if (st != HC_OK) return st;
  int64_t end = dim;                           // behind the rows along the shorter stride
  const bool heads_first = t.n_tokens <= 1 || (t.n_heads > 1 && t.head <= t.token);
  for (int i = 0; i < 2; ++i) {
    const bool heads = heads_first == (i == 0);
    const int64_t n = heads ? t.n_heads : t.n_tokens, stride = heads ? t.head : t.token;
    if (n <= 1) continue;
    if (stride < end) return fail(c, HC_E_INVAL, "%s: rows overlap", t.name);
    end += stride > (INT64_MAX - end) / n ? INT64_MAX - end : (n - 1) * stride;
  }
  return HC_OK;
}

inline hc_status check_scale(hc_ctx *c, float scale) {
  if (!(scale >= 0.f) || !std::isfinite(scale * kLog2E))
    return fail(c, HC_E_INVAL, "softmax_scale must be finite (times log2 e too) and not negative");
  return HC_OK;
}

inline hc_status check_parts(hc_ctx *c, const char *name, const int32_t *cu, int n_tokens, int n_seqs) {
  if (!cu && n_tokens % n_seqs != 0)
    return fail(c, HC_E_INVAL, "%s is NULL, and %d tokens are no %d equal parts", name, n_tokens, n_seqs);
  if (cu && !aligned4(cu)) return fail(c, HC_E_INVAL, "%s must be 4-byte aligned", name);
  return HC_OK;
}

inline float scale_log2(float scale, int head_dim) {
  return (scale > 0.f ? scale : 1.0f / std::sqrt((float)head_dim)) * kLog2E;
}

// Units of R rows that the sequences of a call can have: whole ones, and a partial one each
// (exactly that many where all sequences are alike).
inline int64_t unit_room(int64_t n_tokens, int64_t n_seqs, int64_t group, int R, bool alike) {
  if (alike || n_seqs == 1) return n_seqs * ((n_tokens / n_seqs * group + R - 1) / R);
  return n_tokens * group / R + std::min(n_seqs, n_tokens);
}

// Key ranges per unit.  A launch of fewer work groups than the card runs at once leaves CUs
// idle, so key tiles are shared out until about `want` groups run, but no range is
// shorter than `least` tiles: a partial result costs a write, a read and a merge launch.
inline void choose_split(SeqArgs &a, int64_t keys, int64_t want, int64_t least, int64_t most) {
  const int64_t units = (int64_t)a.tiles * a.kv_heads, tiles = (keys + kSeqKeys - 1) / kSeqKeys;
  const int64_t cuts = std::min({want / std::max<int64_t>(units, 1), tiles / least, most});
  a.n_split = cuts < 2 || !good_grid(units * cuts) ? 1 : (int32_t)cuts;
}

// 128-dim heads: waves of 64 rows, which run the matrix cores better but start slowly and hide
// nothing of it (one wave per SIMD), or of 32.  9360 rows of 12 heads (900 work groups) over 256, 512 and
// 1024 keys: 37, 50 and 75 us against 33, 55 and 95; 1024 rows (96 groups, a
// part of the card) over 512, 1024 and 2048 keys: 20, 27 and 34 us against 18, 25 and 36.
inline bool wide_rows(const SeqArgs &a, int64_t keys) {
  return keys >= ((int64_t)a.tiles * a.kv_heads * a.n_split >= 256 ? 384 : 1536);
}

// Wide kernel, units that take alike (one sequence without a mask, or a window that is shorter than the sequences): two work
// groups per CU make 512 places for them.  What is left over after whole rounds would run alone, each unit on a place of its
// own; instead those units are cut so that their pieces fill the places again: 588 units
// (6200 rows of 12 heads) over 32760 keys without this took as long as 1024 would.
inline void cut_last_round(SeqArgs &a, int64_t keys, bool alike) {
  constexpr int64_t places = 512;
  const int64_t units = seq_units(a), over = units % places;
  if (!a.wide || a.n_split != 1 || !alike || units < places || over == 0) return;
  const int64_t tiles = (keys + kSeqKeys - 1) / kSeqKeys;
  // rounds of pieces, in units, and what a cut costs: about 8 tiles for the start and end of a
  // piece and its partial result
  auto cost = [&](int64_t p) {
    return (double)((over * p + places - 1) / places) * (1.0 / p + (p > 1 ? 8.0 / tiles : 0.0));
  };
  int64_t best = 1;
  for (int64_t p = 2; p <= 8; ++p)
    if (cost(p) < cost(best)) best = p;
  if (best == 1) return;
  a.whole = (int32_t)(units - over);
  a.n_split = (int32_t)best;
}

inline hc_status check_workspace(hc_ctx *c, const void *p, int64_t bytes, int64_t needed) {
  if (needed == 0) return HC_OK;
  if (!p || !aligned16(p) || bytes < needed)
    return fail(c, HC_E_INVAL, "this call needs a 16-byte aligned workspace of %lld bytes", (long long)needed);
  return HC_OK;
}

inline int64_t part_bytes(const SeqArgs &a, int head_dim, int rows, bool logs = false) {
  return seq_cut_units(a) * (16 + a.n_split * seq_part_floats(rows, head_dim, logs) * 4);
}

inline void use_workspace(SeqArgs &a, void *p) {
  a.head = (int32_t *)p;
  a.part = (float *)((char *)p + seq_cut_units(a) * 16);
}

// --- rotary positions -------------------------------------------------------------------
// Types, axes and positions of a rotation; fills `a` but for its tensors and turns.  none_given: positions of no tokens may
// be NULL with any axes and grid, as the address of an empty tensor of them is.
inline hc_status check_rotation(hc_ctx *c, const hc_rotate_args *p, bool none_given, RotateArgs &a) {
  if (p->head_dim < 8 || p->head_dim > kRotMaxDim || p->head_dim % 8 != 0)
    return fail(c, HC_E_INVAL, "head_dim must be a multiple of 8 up to %d", kRotMaxDim);
  for (int type : {p->x_type, p->out_type})
    if (type != HC_BF16 && type != HC_F32) return fail(c, HC_E_INVAL, "types must be HC_BF16 or HC_F32");
  if (p->n_axes < 1 || p->n_axes > kRotMaxAxes) return fail(c, HC_E_INVAL, "n_axes must be 1 to %d", kRotMaxAxes);
  if (!(p->theta > 0) || !std::isfinite(p->theta)) return fail(c, HC_E_INVAL, "theta must be positive and finite");
  a = RotateArgs{};
  int rot = 0;
  for (int i = 0; i < p->n_axes; ++i) {
    if (p->axis_dims[i] < 0 || p->axis_dims[i] > p->head_dim || p->axis_dims[i] % 2 != 0)
      return fail(c, HC_E_INVAL, "axis_dims[%d] must be even and between 0 and head_dim", i);
    rot += p->axis_dims[i];
    a.axis_end[i] = rot / 2;
  }
  if (rot < 16 || rot > p->head_dim || rot % 16 != 0)
    return fail(c, HC_E_INVAL, "axis_dims must add up to a multiple of 16 up to head_dim");
  if (p->positions) {
    if (!aligned4(p->positions)) return fail(c, HC_E_INVAL, "positions must be 4-byte aligned");
  } else if (p->n_tokens > 0 || !none_given) {
    if (p->n_axes != 3 || p->grid_h < 1 || p->grid_w < 1)
      return fail(c, HC_E_INVAL, "positions from the grid need three axes, grid_h and grid_w");
    const int64_t frames = p->n_tokens / ((int64_t)p->grid_h * p->grid_w) + 1;
    if (p->frame0 + frames > INT32_MAX) return fail(c, HC_E_INVAL, "frame0 is too large");
  }
  a.rot = rot;
  return HC_OK;
}

// What the kernels need besides: the angle per position step of every pair.
inline hc_status plan_rotation(hc_ctx *c, const hc_rotate_args *p, RotateArgs &a) {
  a.positions = p->positions;
  a.n_tokens = p->n_tokens; a.head_dim = p->head_dim;
  a.n_axes = p->n_axes;
  a.grid_h = p->grid_h; a.grid_w = p->grid_w; a.frame0 = p->frame0;
  a.sign = p->inverse ? -1.f : 1.f;
  // theta^(-2 j / m) / (2 pi), by repeated products (63 roundings of 2^-53 at most)
  const double per_turn = 0.15915494309189533577;
  for (int i = 0, pair = 0; i < p->n_axes; ++i) {
    const int m = p->joint ? a.rot : p->axis_dims[i];
    const double step = m > 0 ? std::pow(p->theta, -2.0 / m) : 1.0;
    for (int j = 0; j < p->axis_dims[i] / 2; ++j, ++pair) {
      a.turns[pair] = (p->joint ? pair : j) == 0 ? per_turn : a.turns[pair - 1] * step;
      if (!std::isfinite(a.turns[pair] * 0x1p31)) return fail(c, HC_E_INVAL, "theta is too small");
    }
  }
  return HC_OK;
}

}  // namespace hc
