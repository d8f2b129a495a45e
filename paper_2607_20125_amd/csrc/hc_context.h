// The context behind the C ABI, and what every entry point does with it: error
// messages, checked HIP calls, timed launches.  Included by the files that hold
// entry points (hc_runtime.cpp, hc_ops.cpp).
#pragma once

#include <cstdarg>
#include <cstdio>
#include <new>
#include <string>
#include <vector>

#include "hc_internal.h"
#include "hc_plan.h"

namespace hc {

struct DevBuf {
  void *p = nullptr;
  size_t bytes = 0;
};

struct Layer {
  bool has_types = false;
  std::vector<uint8_t> types;
  std::vector<int32_t> slot;
  std::vector<int> sd_heads, sp_heads, g_heads;
  int64_t cur_block = -1;
  // the compact buffers: parts of one allocation, `kv`
  DevBuf kv, k_sd, v_sd, k_g, v_g, k_sp, v_sp;
  // dense work units and, behind them, combine items of the current plan
  DevBuf plan;
  const DenseUnit *units = nullptr;
  const CombineItem *comb = nullptr;
  int n_units = 0, n_comb = 0;
  bool plan_wide = false;      // 128-dim heads: the units run on waves of 64 queries
  int64_t plan_slots = 0;      // partial slots that the units write
  int plan_nv = -1;            // valid window blocks the plan was built for
  bool plan_used = false;      // launches may still read the plan's memory
  hipStream_t kv_stream = nullptr;   // the stream that last wrote the compact buffers
  int static_nv = -1;          // window fill that `chosen` is for
  StaticChoice chosen{};       // the device-built work list
  int sp_split = 1;            // key-frame split of the Spatial work (full window)
};

struct EventPair {
  hipEvent_t a, b;
};

}  // namespace hc

struct hc_ctx {
  hc_config cfg{};
  int device = 0;
  float scale = 0.f;
  int L = 0, P = 0;
  hc::SpatialGeom geo{};          // frame storage of the Spatial buffers (centred window)
  int64_t sd_keys = 0, g_keys = 0, sp_keys = 0;
  std::vector<hc::Layer> layers;
  std::string err;
  bool profile = false;
  std::vector<hc::EventPair> pending[HC_K_COUNT];
  std::vector<hc::EventPair> pool;
  double prof_ms[HC_K_COUNT] = {};
  int64_t prof_n[HC_K_COUNT] = {};
  hc::DevBuf part;                 // partial-result slots shared by all layers
  int64_t part_slots = 0;
  hc::DevBuf sp_part, sp_ml;       // Spatial split partials shared by all layers
  int64_t sp_part_rows = 0;
  int n_cu = 0;                // compute units of the device
  // cell variant of the Spatial path (cfg.spatial_cell > 0)
  hc::CellTables cells;
  hc::DevBuf cell_off_d, qmap_d;   // cells.off and cells.qmap on the device
  // device memory of hc_classify_heads, allocated (and zeroed) by the first call
  // and reused by the next ones: the window in Global and in Spatial layout, the
  // four proxy outputs, the block partials, the work lists, the token statistics
  hc::DevBuf cls_k, cls_v, cls_pk, cls_pv, cls_o[4], cls_part, cls_units, cls_comb, cls_tok;
  int cls_n_units = 0, cls_n_comb = 0;
  bool cls_wide = false;       // 128-dim heads: the sweep runs on waves of 64 queries
  bool cls_done = false;       // cls_o holds the outputs of a successful classification
  void *scratch = nullptr;     // this device's fixed scratch (hc_attention_static)
  // the last choices of hc_attention_static: layers with as many heads of each kind
  // at the same window fill share one
  struct {
    int n_g, n_sd, nv;
    bool merged;
    hc::StaticChoice choice;
  } static_memo[16];
  int static_memos = 0;        // choices made
};

namespace hc {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline hc_status fail(hc_ctx *c, hc_status s, const char *fmt, ...) {
  if (c) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
      c->err = buf;
    } catch (const std::bad_alloc &) {
      c->err.clear();
    }
  }
  return s;
}

// Ends the functions that allocate host memory: nothing is thrown across the ABI.
#define HC_NO_HOST_MEMORY(ctx) \
  catch (const std::bad_alloc &) { return fail(ctx, HC_E_NOMEM, "out of host memory"); }

// A failed HIP call stays the thread's last error until it is read, and the next
// launch would take it for its own: every failure that is reported or passed over
// here is read off first.
#define HC_HIP(ctx, call)                                                               \
  do {                                                                                  \
    hipError_t e_ = (call);                                                             \
    if (e_ != hipSuccess) {                                                             \
      (void)hipGetLastError();                                                          \
      return fail(ctx, e_ == hipErrorOutOfMemory ? HC_E_NOMEM : HC_E_DEVICE, "%s: %s", \
                  #call, hipGetErrorString(e_));                                        \
    }                                                                                   \
  } while (0)

// --- profiling ----------------------------------------------------------------
inline hc_status prof_begin(hc_ctx *c, hipStream_t s, EventPair *ep) {
  if (!c->profile) return HC_OK;
  if (c->pool.empty()) {
    EventPair p;
    HC_HIP(c, hipEventCreate(&p.a));
    const hipError_t e = hipEventCreate(&p.b);
    if (e != hipSuccess) {
      (void)hipEventDestroy(p.a);
      (void)hipGetLastError();
      return fail(c, HC_E_DEVICE, "hipEventCreate: %s", hipGetErrorString(e));
    }
    c->pool.push_back(p);
  }
  *ep = c->pool.back();
  c->pool.pop_back();
  HC_HIP(c, hipEventRecord(ep->a, s));
  return HC_OK;
}

inline hc_status prof_end(hc_ctx *c, hipStream_t s, int kind, const EventPair &ep) {
  if (!c->profile) return HC_OK;
  HC_HIP(c, hipEventRecord(ep.b, s));
  c->pending[kind].push_back(ep);
  return HC_OK;
}

template <class F>
hc_status timed_launch(hc_ctx *c, hipStream_t s, int kind, F &&launch) {
  EventPair ep{};
  hc_status st = prof_begin(c, s, &ep);
  if (st != HC_OK) return st;
  hipError_t e = launch();
  if (e != hipSuccess) return fail(c, HC_E_DEVICE, "kernel launch: %s", hipGetErrorString(e));
  return prof_end(c, s, kind, ep);
}

}  // namespace hc
