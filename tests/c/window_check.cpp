// Checks of the entry points of a model with a sliding window (hc_window.cpp) on the CPU: what they refuse, what they
// hand to the launchers, and the rooms they plan.  Compiled with hc_runtime.cpp against the HIP runtime of
// fake_hip.h; one check per run, by name.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <functional>
#include <limits>
#include <string>

#define hipSetDevice ignored_set_device       // (fake_hip.h's looks at no device)
#include "fake_hip.h"
#undef hipSetDevice
#include "hc_window.h"
#include "headcast.h"

using namespace hc;

namespace {
int fails = 0;
#define CHECK(cond)                                                           \
  do {                                                                        \
    if (!(cond)) {                                                            \
      std::fprintf(stderr, "check failed: %s (line %d)\n", #cond, __LINE__); \
      ++fails;                                                                \
    }                                                                         \
  } while (0)

int device_now = 0, device_in_launch = -1;
NormArgs normed;
PagedRowsArgs stored;
SeqArgs attended;
GradArgs graded;
bool decoded = false, merged = false, backward = false;
hipError_t launch_result = hipSuccess;
hipError_t launched() {
  ++fake::launches;
  device_in_launch = device_now;
  return launch_result;
}
}  // namespace

extern "C" {
hipError_t hipGetDevice(int *d) { *d = device_now; return hipSuccess; }
hipError_t hipSetDevice(int d) { device_now = d; return hipSuccess; }
}

namespace hc {
hipError_t launch_norm(const NormArgs &a, int, int, bool, hipStream_t) { normed = a; backward = false; return launched(); }
hipError_t launch_norm_backward(const NormArgs &a, int, int, bool, hipStream_t) { normed = a; backward = true; return launched(); }
hipError_t launch_paged_append(const PagedRowsArgs &a, hipStream_t) { stored = a; return launched(); }
hipError_t launch_window(const SeqArgs &a, int, hipStream_t) { attended = a; decoded = merged = false; return launched(); }
hipError_t launch_paged_decode(const SeqArgs &a, int, hipStream_t) {
  attended = a;
  decoded = true;
  merged = false;
  return launched();
}
hipError_t launch_seq_merge(const SeqArgs &, int, int, hipStream_t) { merged = true; return launched(); }
hipError_t launch_grad64(const GradArgs &a, hipStream_t) { graded = a; return launched(); }
hipError_t launch_grad128(const GradArgs &a, hipStream_t) { graded = a; return launched(); }
}  // namespace hc

namespace {

struct Ctx {
  hc_ctx *c = nullptr;
  Ctx() {
    hc_config cfg;
    hc_config_default(&cfg);
    CHECK(hc_create(&cfg, 0, &c) == HC_OK);
  }
  ~Ctx() { hc_destroy(c); }
};

alignas(16) char memory[8192];
void *const at = memory;
const int32_t *const iat = (const int32_t *)memory;

// Every change of a good call must be refused, with a message and without a launch.
template <class Args>
void refuses(hc_ctx *c, const Args &good, std::initializer_list<std::function<void(Args &)>> changes,
             const std::function<hc_status(const Args &)> &call) {
  CHECK(call(good) == HC_OK);
  int i = 0;
  for (const auto &change : changes) {
    Args a = good;
    change(a);
    const int before = fake::launches;
    const hc_status st = call(a);
    if (st != HC_E_INVAL || fake::launches != before || !*hc_last_error(c)) {
      std::fprintf(stderr, "change %d: status %d, message '%s'\n", i, (int)st, hc_last_error(c));
      ++fails;
    }
    ++i;
  }
}

// --- norm -------------------------------------------------------------------------------------
struct Norm {
  hc_norm_args a;
  hc_norm_tensor t[2];
  hc_norm_grad_tensor g[2];
  int n;
  void *workspace;
  int64_t bytes;
};
Norm good_norm() {
  Norm r{};
  hc_rotate_args &a = r.a.rotate;
  a.n_tokens = 100; a.head_dim = 128; a.n_axes = 3;
  a.axis_dims[0] = 44; a.axis_dims[1] = a.axis_dims[2] = 42;
  a.grid_h = 5; a.grid_w = 4; a.theta = 1e4;
  r.a.eps = 1e-6f;
  r.t[0] = {at, memory + 2048, memory + 4096, 12 * 128, 128, 128, 100 * 128, 12};
  r.t[1] = {at, at, nullptr, 4 * 128, 128, 4 * 128, 128, 4};
  r.g[0] = {at, memory + 2048, memory + 4096, memory + 3584, (float *)(memory + 6144), 12 * 128, 128, 128, 100 * 128, 12 * 128, 128, 12};
  r.g[1] = {at, memory + 1024, nullptr, memory + 1024, nullptr, 4 * 128, 128, 4 * 128, 128, 4 * 128, 128, 4};
  r.n = 2;
  r.workspace = at;
  r.bytes = INT64_MAX;
  return r;
}

void norm_refusals() {
  Ctx x;
  const float nan = std::numeric_limits<float>::quiet_NaN();
  const std::function<hc_status(const Norm &)> forward = [&](const Norm &r) { return hc_norm_rotate(x.c, &r.a, r.t, r.n, nullptr); };
  const std::function<hc_status(const Norm &)> back = [&](const Norm &r) {
    return hc_norm_rotate_backward(x.c, &r.a, r.g, r.n, r.workspace, r.bytes, nullptr);
  };
  for (const auto &call : {forward, back})
    refuses<Norm>(x.c, good_norm(), {
        [](Norm &r) { r.n = 0; }, [](Norm &r) { r.n = 3; }, [](Norm &r) { r.a.rotate.n_tokens = -1; },
        [](Norm &r) { r.a.rotate.head_dim = 132; }, [](Norm &r) { r.a.rotate.head_dim = 264; }, [](Norm &r) { r.a.rotate.x_type = 2; },
        [](Norm &r) { r.a.rotate.out_type = -1; }, [](Norm &r) { r.a.weight_type = 7; }, [](Norm &r) { r.a.eps = -1; },
        [nan](Norm &r) { r.a.eps = nan; }, [](Norm &r) { r.a.eps = INFINITY; }, [](Norm &r) { r.a.rotate.n_axes = 0; },
        [](Norm &r) { r.a.rotate.axis_dims[0] = 43; }, [](Norm &r) { r.a.rotate.axis_dims[0] = 60; }, [](Norm &r) { r.a.rotate.theta = 0; },
        [](Norm &r) { r.a.rotate.theta = INFINITY; }, [](Norm &r) { r.a.rotate.grid_h = 0; }, [](Norm &r) { r.a.rotate.frame0 = INT32_MAX; },
        [](Norm &r) { r.a.rotate.positions = (const int32_t *)(memory + 2); },
        [](Norm &r) { r.t[1].n_heads = r.g[1].n_heads = 0; }, [](Norm &r) { r.t[0].n_heads = r.g[0].n_heads = 70000; },
        [](Norm &r) { r.t[0].x = r.g[0].x = nullptr; }, [](Norm &r) { r.t[0].x = r.g[0].x = memory + 8; },
        [](Norm &r) { r.t[0].weight = r.g[0].weight = memory + 4; }, [](Norm &r) { r.t[0].x_token = r.g[0].x_token = 12 * 128 + 4; },
    }, call);
  refuses<Norm>(x.c, good_norm(), {
      [](Norm &r) { r.t[0].out = nullptr; }, [](Norm &r) { r.t[0].out_head = 99 * 128; }, [](Norm &r) { r.t[0].out_token = 0; },
      [](Norm &r) { r.t[1].out_token = 8 * 128; }, [](Norm &r) { r.a.rotate.out_type = HC_F32; },        // in place
  }, forward);
  refuses<Norm>(x.c, good_norm(), {
      [](Norm &r) { r.g[0].dout = nullptr; }, [](Norm &r) { r.g[0].dx = nullptr; }, [](Norm &r) { r.g[0].dx_token = 0; },
      [](Norm &r) { r.g[0].dweight = (float *)(memory + 4); }, [](Norm &r) { r.workspace = nullptr; }, [](Norm &r) { r.bytes = 100; },
      [](Norm &r) { r.workspace = memory + 4; },
      [](Norm &r) { r.g[1].dx_token = 8 * 128; }, [](Norm &r) { r.a.rotate.out_type = HC_F32; },         // in the place of dout
      [](Norm &r) { r.g[0].dx = at; r.g[0].dx_token = 24 * 128; },                                       // of x
  }, back);
  const Norm r = good_norm();
  CHECK(hc_norm_rotate(nullptr, &r.a, r.t, 2, nullptr) == HC_E_INVAL && hc_norm_rotate(x.c, nullptr, r.t, 2, nullptr) == HC_E_INVAL);
  CHECK(hc_norm_rotate(x.c, &r.a, nullptr, 2, nullptr) == HC_E_INVAL);
  CHECK(hc_norm_rotate_backward(nullptr, &r.a, r.g, 2, at, 1 << 30, nullptr) == HC_E_INVAL);
  int64_t bytes = -1;
  CHECK(hc_norm_rotate_workspace(x.c, &r.a, r.g, 2, nullptr) == HC_E_INVAL);
  CHECK(hc_norm_rotate_workspace(x.c, &r.a, r.g, 2, &bytes) == HC_OK && bytes > 0);
  CHECK(bytes == (norm_parts(normed, 0) + norm_parts(normed, 1)) * 128 * 4);
  Norm s = r;
  s.bytes = bytes - 1;
  CHECK(back(s) == HC_E_INVAL);
  s.bytes = bytes;
  CHECK(back(s) == HC_OK && backward);
  // no tokens: nothing to norm, and the weights' gradients are written
  Norm none = r;
  none.a.rotate.n_tokens = 0;
  none.workspace = nullptr;
  none.bytes = 0;
  const int before = fake::launches;
  CHECK(forward(none) == HC_OK && fake::launches == before);
  CHECK(back(none) == HC_OK && fake::launches == before + 1 && normed.groups == 0);
  // every token and head has a thread, and lanes are powers of two up to 32
  for (int halves = 0; halves < 2; ++halves)
    for (int dim = 16; dim <= 256; dim += 8)
      for (int n : {1, 7, 100, 5000, 100000}) {
        Norm q = r;
        q.a.rotate.n_tokens = n; q.a.rotate.head_dim = dim; q.a.rotate.halves = halves;
        q.a.rotate.axis_dims[0] = 16; q.a.rotate.axis_dims[1] = q.a.rotate.axis_dims[2] = 0;
        q.t[0].out_token = 12 * 256; q.t[0].out_head = 256;
        q.t[0].out = memory + 2048; q.t[1].out = memory + 2560;
        q.t[1].out_token = 4 * 256; q.t[1].out_head = 256;
        CHECK(forward(q) == HC_OK);
        CHECK(normed.lane_bits <= 5 && (1 << normed.lane_bits) >= norm_items(normed.rotate, halves));
        CHECK((int64_t)normed.groups * (kNormThreads >> normed.lane_bits) >= n);
        for (int i = 0; i < 2; ++i) CHECK(normed.t[i].cuts >= 1 && normed.t[i].cuts <= normed.t[i].n_heads);
      }
}

void no_tokens() {
  Ctx x;
  Norm r = good_norm();
  r.a.rotate.n_axes = 1;
  r.a.rotate.axis_dims[0] = 128; r.a.rotate.axis_dims[1] = r.a.rotate.axis_dims[2] = 0;
  CHECK(hc_norm_rotate(x.c, &r.a, r.t, r.n, nullptr) == HC_E_INVAL);         // neither positions nor a grid
  r.a.rotate.n_tokens = 0;
  CHECK(hc_norm_rotate(x.c, &r.a, r.t, r.n, nullptr) == HC_OK);
  CHECK(hc_norm_rotate_backward(x.c, &r.a, r.g, r.n, nullptr, 0, nullptr) == HC_OK && normed.groups == 0);
}

// --- pages ------------------------------------------------------------------------------------
struct Paged {
  hc_pages p;
  hc_page_table t;
  hc_qcache_rows r;
  hc_paged_args a;
};
Paged good_paged() {
  Paged x{};
  x.p = {at, memory + 4096, 16 * 128, 128, 64, 16 * 128, 64, 16 * 64, 9, 16, 2, 64};
  x.t = {iat, 5, 3, 5};
  x.r = {memory + 2048, memory + 2560, 128, 64, 128, 64, 9, iat, nullptr};
  x.a.q = memory + 2048; x.a.out = memory + 2560;
  x.a.q_token = x.a.out_token = 256; x.a.q_head = x.a.out_head = 64;
  x.a.n_tokens = 6; x.a.n_heads = 4; x.a.causal_block = 1; x.a.kv_len = iat;
  return x;
}

void paged_refusals() {
  Ctx x;
  const std::function<hc_status(const Paged &)> append = [&](const Paged &q) { return hc_paged_append(x.c, &q.p, &q.t, &q.r, nullptr); };
  const std::function<hc_status(const Paged &)> attend = [&](const Paged &q) { return hc_paged_attention(x.c, &q.p, &q.t, &q.a, nullptr); };
  for (const auto &call : {append, attend})
    refuses<Paged>(x.c, good_paged(), {
        [](Paged &q) { q.p.k = nullptr; }, [](Paged &q) { q.p.v = memory + 8; }, [](Paged &q) { q.p.n_pages = 0; },
        [](Paged &q) { q.p.page_tokens = 8; }, [](Paged &q) { q.p.page_tokens = 48; }, [](Paged &q) { q.p.page_tokens = 1 << 17; },
        [](Paged &q) { q.p.n_heads = 0; }, [](Paged &q) { q.p.head_dim = 96; }, [](Paged &q) { q.p.k_page = 100; },
        [](Paged &q) { q.p.v_token = -64; }, [](Paged &q) { q.p.k_head = 12; }, [](Paged &q) { q.t.table = nullptr; },
        [](Paged &q) { q.t.table = (const int32_t *)(memory + 2); }, [](Paged &q) { q.t.n_seqs = 0; }, [](Paged &q) { q.t.max_pages = 0; },
        [](Paged &q) { q.t.stride = 4; }, [](Paged &q) { q.t.max_pages = INT32_MAX; q.t.stride = INT32_MAX; },
        [](Paged &q) { q.r.n_tokens = q.a.n_tokens = -1; }, [](Paged &q) { q.r.n_tokens = q.a.n_tokens = 10; },
        [](Paged &q) { q.r.cu_seqlens = q.a.cu_seqlens = (const int32_t *)(memory + 2); },
    }, call);
  refuses<Paged>(x.c, good_paged(), {
      [](Paged &q) { q.r.k = nullptr; }, [](Paged &q) { q.r.v = memory + 4; }, [](Paged &q) { q.r.k_token = 12; },
      [](Paged &q) { q.r.start = nullptr; }, [](Paged &q) { q.r.start = (const int32_t *)(memory + 2); },
      [](Paged &q) { q.p.k_page = 15 * 128; }, [](Paged &q) { q.p.v_head = 0; }, [](Paged &q) { q.p.k_token = 56; },   // rows that overlap
      [](Paged &q) { q.p.v_token = 0; },
  }, append);
  refuses<Paged>(x.c, good_paged(), {
      [](Paged &q) { q.a.n_heads = 3; }, [](Paged &q) { q.a.n_heads = 0; }, [](Paged &q) { q.a.causal_block = -1; },
      [](Paged &q) { q.a.window = -1; }, [](Paged &q) { q.a.sinks = -1; }, [](Paged &q) { q.a.max_kv = -1; },
      [](Paged &q) { q.a.causal_block = 0; q.a.window = 5; }, [](Paged &q) { q.a.softmax_scale = NAN; },
      [](Paged &q) { q.a.softmax_scale = 3e38f; }, [](Paged &q) { q.a.kv_len = nullptr; }, [](Paged &q) { q.a.q = nullptr; },
      [](Paged &q) { q.a.kv_len = (const int32_t *)(memory + 2); }, [](Paged &q) { q.a.out = memory + 2; }, [](Paged &q) { q.a.out_token = 128; },
      [](Paged &q) { q.a.n_tokens = INT32_MAX; q.a.cu_seqlens = iat; },
  }, attend);
  Paged q = good_paged();
  CHECK(hc_paged_append(nullptr, &q.p, &q.t, &q.r, nullptr) == HC_E_INVAL && hc_paged_append(x.c, nullptr, &q.t, &q.r, nullptr) == HC_E_INVAL);
  CHECK(hc_paged_append(x.c, &q.p, nullptr, &q.r, nullptr) == HC_E_INVAL && hc_paged_append(x.c, &q.p, &q.t, nullptr, nullptr) == HC_E_INVAL);
  CHECK(hc_paged_attention(nullptr, &q.p, &q.t, &q.a, nullptr) == HC_E_INVAL && hc_paged_attention(x.c, &q.p, &q.t, nullptr, nullptr) == HC_E_INVAL);
  // rows that overlap may be read, and one row stored everywhere
  q.p.k_page = 0;
  CHECK(attend(q) == HC_OK && decoded);
  q = good_paged();
  q.r.k_token = 0;
  CHECK(append(q) == HC_OK && stored.page_shift == 4);
  // a long table needs a workspace, and no device memory is looked at for its size
  int64_t bytes = -1;
  q.t.max_pages = 20000;
  q.t.stride = 20000;
  hc_pages none = q.p;
  none.k = none.v = nullptr;
  hc_page_table empty = q.t;
  empty.table = nullptr;
  CHECK(hc_paged_workspace(x.c, &none, &empty, &q.a, &bytes) == HC_OK && bytes > 0);
  CHECK(hc_paged_workspace(x.c, &none, &empty, &q.a, nullptr) == HC_E_INVAL);
  CHECK(attend(q) == HC_E_INVAL);
  q.a.workspace = memory + 1024;
  q.a.workspace_bytes = bytes - 1;
  CHECK(attend(q) == HC_E_INVAL);
  q.a.workspace_bytes = bytes;
  CHECK(attend(q) == HC_OK && decoded && merged);
  // a window is shorter than the table: fewer ranges
  q.a.window = 100;
  CHECK(hc_paged_workspace(x.c, &q.p, &q.t, &q.a, &bytes) == HC_OK && bytes == 0);
  Paged nothing = good_paged();
  nothing.r.n_tokens = nothing.a.n_tokens = 0;
  nothing.r.k = nothing.r.v = nullptr;
  const int before = fake::launches;
  CHECK(append(nothing) == HC_OK && attend(nothing) == HC_OK && fake::launches == before);
}

// --- packed sequences and their gradients -------------------------------------------------------
hc_window_grad_args good_window() {
  hc_window_grad_args g{};
  hc_window_args &p = g.forward;
  p.q = p.k = p.v = at;
  p.out = memory + 2048;
  p.lse = (float *)(memory + 4096);
  p.q_token = p.out_token = 8 * 64; p.k_token = p.v_token = 2 * 64;
  p.q_head = p.k_head = p.v_head = p.out_head = 64;
  p.n_tokens = 40; p.n_keys = 40; p.n_seqs = 3;
  p.n_heads = 8; p.n_kv_heads = 2; p.head_dim = 64; p.causal_block = 1; p.window = 7; p.sinks = 2;
  p.cu_q = iat;
  g.dout = memory + 1024;
  g.dq = memory + 5120; g.dk = memory + 6144; g.dv = memory + 7168;
  g.dout_token = g.dq_token = 8 * 64; g.dk_token = g.dv_token = 2 * 64;
  g.dout_head = g.dq_head = g.dk_head = g.dv_head = 64;
  g.workspace = memory + 512;
  g.workspace_bytes = INT64_MAX;
  return g;
}

void window_refusals() {
  Ctx x;
  using G = hc_window_grad_args;
  const std::function<hc_status(const G &)> forward = [&](const G &g) { return hc_window_attention(x.c, &g.forward, nullptr); };
  const std::function<hc_status(const G &)> back = [&](const G &g) { return hc_window_attention_backward(x.c, &g, nullptr); };
  for (const auto &call : {forward, back})
    refuses<G>(x.c, good_window(), {
        [](G &g) { g.forward.n_tokens = -1; }, [](G &g) { g.forward.n_keys = -1; }, [](G &g) { g.forward.n_keys = 41; },
        [](G &g) { g.forward.n_seqs = 0; }, [](G &g) { g.forward.n_heads = 7; }, [](G &g) { g.forward.n_kv_heads = 0; },
        [](G &g) { g.forward.n_heads = 0; }, [](G &g) { g.forward.head_dim = 96; }, [](G &g) { g.forward.causal_block = -1; },
        [](G &g) { g.forward.window = -1; }, [](G &g) { g.forward.sinks = -1; }, [](G &g) { g.forward.causal_block = 0; },
        [](G &g) { g.forward.softmax_scale = -1; }, [](G &g) { g.forward.softmax_scale = NAN; },
        [](G &g) { g.forward.softmax_scale = 3e38f; }, [](G &g) { g.forward.cu_q = nullptr; },
        [](G &g) { g.forward.cu_q = (const int32_t *)(memory + 1); }, [](G &g) { g.forward.cu_k = (const int32_t *)(memory + 2); },
        [](G &g) { g.forward.lse = (float *)(memory + 2); }, [](G &g) { g.forward.q = nullptr; }, [](G &g) { g.forward.k = nullptr; },
        [](G &g) { g.forward.v = memory + 8; }, [](G &g) { g.forward.out = nullptr; }, [](G &g) { g.forward.k_token = 100; },
        [](G &g) { g.forward.v_head = -64; }, [](G &g) { g.forward.n_tokens = g.forward.n_keys = INT32_MAX; },
        [](G &g) { g.forward.cu_k = iat; g.forward.n_keys = INT32_MAX; },
    }, call);
  refuses<G>(x.c, good_window(), {[](G &g) { g.forward.out_head = 56; }, [](G &g) { g.forward.out_token = 0; }}, forward);
  refuses<G>(x.c, good_window(), {
      [](G &g) { g.forward.lse = nullptr; }, [](G &g) { g.forward.out = at; }, [](G &g) { g.dout = nullptr; }, [](G &g) { g.dout_token = 100; },
      [](G &g) { g.dq = memory + 4; }, [](G &g) { g.dk = nullptr; }, [](G &g) { g.dv = nullptr; }, [](G &g) { g.dq_token = 0; },
      [](G &g) { g.dk_head = 56; }, [](G &g) { g.dv_token = 64; }, [](G &g) { g.workspace = nullptr; }, [](G &g) { g.workspace_bytes = 10; },
      [](G &g) { g.workspace = memory + 4; }, [](G &g) { g.forward.q_token = 1 << 24; }, [](G &g) { g.forward.v_token = 1 << 24; },
      [](G &g) { g.dout_token = (int64_t)1 << 40; }, [](G &g) { g.forward.softmax_scale = 1e-32f; },
  }, back);
  G g = good_window();
  CHECK(hc_window_attention(nullptr, &g.forward, nullptr) == HC_E_INVAL && hc_window_attention(x.c, nullptr, nullptr) == HC_E_INVAL);
  CHECK(hc_window_attention_backward(nullptr, &g, nullptr) == HC_E_INVAL && hc_window_attention_backward(x.c, nullptr, nullptr) == HC_E_INVAL);
  int64_t bytes = -1;
  CHECK(hc_window_workspace(x.c, &g.forward, nullptr) == HC_E_INVAL && hc_window_backward_workspace(x.c, &g, nullptr) == HC_E_INVAL);
  CHECK(hc_window_backward_workspace(x.c, &g, &bytes) == HC_OK && bytes >= 40 * 8 * 2 * 4);
  g.workspace_bytes = bytes;
  CHECK(back(g) == HC_OK);
  // few rows over many keys: ranges, and a workspace
  g.forward.cu_k = iat;
  g.forward.n_keys = 300000;
  g.forward.window = 0;
  CHECK(hc_window_workspace(x.c, &g.forward, &bytes) == HC_OK && bytes > 0);
  CHECK(forward(g) == HC_E_INVAL);
  g.forward.workspace = memory + 1024;
  g.forward.workspace_bytes = bytes;
  CHECK(forward(g) == HC_OK && merged && attended.n_split > 1 && attended.lse == g.forward.lse);
  // no tokens, no keys
  G none = good_window();
  none.forward.n_tokens = none.forward.n_keys = 0;
  const int before = fake::launches;
  CHECK(forward(none) == HC_OK && back(none) == HC_OK && fake::launches == before);
  // keys that no query can see: their gradients are written
  none.forward.n_keys = 40;
  none.forward.cu_k = iat;
  none.forward.q = none.forward.out = nullptr;
  none.dout = none.dq = nullptr;
  none.forward.lse = nullptr;
  CHECK(forward(none) == HC_OK && fake::launches == before);
  CHECK(back(none) == HC_OK && fake::launches == before + 1 && graded.key_tiles > 0 && graded.seq.tiles == 0);
  // no keys: queries get zeros
  none = good_window();
  none.forward.n_keys = 0;
  none.forward.cu_k = iat;
  none.forward.k = none.forward.v = nullptr;
  none.dk = none.dv = nullptr;
  CHECK(forward(none) == HC_OK && back(none) == HC_OK && graded.key_tiles == 0);
}

// The units that sequences of any lengths need never exceed the room of the launch.
void rooms() {
  Ctx x;
  uint32_t seed = 1;
  auto rnd = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (uint32_t)n); };
  for (int round = 0; round < 2000; ++round) {
    const int n_seqs = 1 + rnd(40), group = 1 + rnd(9), longest = 1 + rnd(400);
    std::vector<int> len[2];
    int total[2] = {0, 0};
    for (int i = 0; i < 2; ++i) {
      len[i].resize(n_seqs);
      for (int &n : len[i]) total[i] += n = rnd(3) ? rnd(longest) : 0;
      if (total[i] == 0) total[i] = len[i][0] = 1;
    }
    auto needed = [&](const std::vector<int> &l, int g, int R) {
      int64_t u = 0;
      for (int n : l) u += (n * g + R - 1) / R;
      return u;
    };
    hc_window_grad_args g = good_window();
    hc_window_args &p = g.forward;
    p.n_seqs = n_seqs; p.n_kv_heads = 1; p.n_heads = group; p.n_tokens = total[0]; p.n_keys = total[1];
    p.cu_k = iat;
    p.q_token = p.out_token = g.dout_token = g.dq_token = 64 * group;
    p.workspace = at;
    p.workspace_bytes = INT64_MAX;
    CHECK(hc_window_attention(x.c, &p, nullptr) == HC_OK && attended.tiles >= needed(len[0], group, kSeqRows));
    CHECK(hc_window_attention_backward(x.c, &g, nullptr) == HC_OK);
    CHECK(graded.seq.tiles >= needed(len[0], 1, kSeqRows) && graded.key_tiles >= needed(len[1], 1, kGradKeys));
    Paged q = good_paged();
    q.p.n_heads = 1;
    q.t.n_seqs = n_seqs;
    q.a.n_heads = group; q.a.n_tokens = total[0]; q.a.cu_seqlens = iat;
    q.a.q_token = q.a.out_token = 64 * group;
    CHECK(hc_paged_attention(x.c, &q.p, &q.t, &q.a, nullptr) == HC_OK);
    CHECK(attended.tiles >= needed(len[0], group, decoded ? kDecodeRows : kSeqRows));
    // equal parts: exactly as many as they need
    p.n_tokens = p.n_keys = n_seqs * longest;
    p.cu_q = p.cu_k = nullptr;
    CHECK(hc_window_attention_backward(x.c, &g, nullptr) == HC_OK);
    CHECK(graded.seq.tiles == n_seqs * ((longest + kSeqRows - 1) / kSeqRows));
    CHECK(graded.key_tiles == n_seqs * ((longest + kGradKeys - 1) / kGradKeys));
  }
}

// Every call launches on its context's device and leaves the caller's current, whatever the launch returns.
void call_devices() {
  Ctx x;
  const Norm r = good_norm();
  const Paged q = good_paged();
  const hc_window_grad_args g = good_window();
  const std::function<hc_status()> calls[] = {
      [&] { return hc_norm_rotate(x.c, &r.a, r.t, r.n, nullptr); },
      [&] { return hc_norm_rotate_backward(x.c, &r.a, r.g, r.n, r.workspace, r.bytes, nullptr); },
      [&] { return hc_paged_append(x.c, &q.p, &q.t, &q.r, nullptr); },
      [&] { return hc_paged_attention(x.c, &q.p, &q.t, &q.a, nullptr); },
      [&] { return hc_window_attention(x.c, &g.forward, nullptr); },
      [&] { return hc_window_attention_backward(x.c, &g, nullptr); },
  };
  for (int current : {1, 0, 5})
    for (hipError_t result : {hipSuccess, hipErrorUnknown}) {
      launch_result = result;
      for (const auto &call : calls) {
        device_now = current;
        device_in_launch = -1;
        CHECK(call() == (result == hipSuccess ? HC_OK : HC_E_DEVICE));
        CHECK(device_in_launch == 0 && device_now == current);
      }
    }
  launch_result = hipSuccess;
  device_now = 0;
}

}  // namespace

int main(int argc, char **argv) {
  const std::string name = argc > 1 ? argv[1] : "";
  if (name == "norm_refusals") norm_refusals();
  else if (name == "no_tokens") no_tokens();
  else if (name == "paged_refusals") paged_refusals();
  else if (name == "window_refusals") window_refusals();
  else if (name == "rooms") rooms();
  else if (name == "call_devices") call_devices();
  else return 2;
  for (const std::string &f : fake::faults) std::fprintf(stderr, "%s\n", f.c_str());
  if (fails || !fake::faults.empty()) return 1;
  std::printf("%s: ok\n", name.c_str());
  return 0;
}
