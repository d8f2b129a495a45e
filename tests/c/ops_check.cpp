// Checks of the entry points beside the routed attention (hc_ops.cpp) on the CPU: what they
// refuse, what they hand to the launchers, and the rooms they plan.  Compiled with
// hc_runtime.cpp against the HIP runtime of fake_hip.h; one check per run, by name.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <functional>
#include <limits>
#include <string>

#include "fake_hip.h"
#include "hc_ops.h"
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
RotateArgs rotated;
QCacheArgs rowed;
SeqArgs attended;
bool decoded = false, merged = false;
hipError_t launch_result = hipSuccess;
hipError_t launched() {
  ++fake::launches;
  device_in_launch = device_now;
  return launch_result;
}
}  // namespace

extern "C" {
hipError_t hipGetDevice(int *d) { *d = device_now; return hipSuccess; }
}

namespace hc {
hipError_t launch_rotate(const RotateArgs &a, int, int, bool, hipStream_t) { rotated = a; return launched(); }
hipError_t launch_qcache_append(const QCacheArgs &a, hipStream_t) { rowed = a; return launched(); }
hipError_t launch_qcache_read(const QCacheArgs &a, hipStream_t) { rowed = a; return launched(); }
hipError_t launch_seq(const SeqArgs &a, int, hipStream_t) { attended = a; decoded = merged = false; return launched(); }
hipError_t launch_decode(const SeqArgs &a, int, hipStream_t) {
  attended = a;
  decoded = true;
  merged = false;
  return launched();
}
hipError_t launch_seq_merge(const SeqArgs &, int, int, hipStream_t) { merged = true; return launched(); }
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

alignas(16) char memory[4096];
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

struct Rot {
  hc_rotate_args a;
  hc_rotate_tensor t[2];
  int n;
};
Rot good_rotate() {
  Rot r{};
  r.a.n_tokens = 100; r.a.head_dim = 128; r.a.n_axes = 3;
  r.a.axis_dims[0] = 44; r.a.axis_dims[1] = r.a.axis_dims[2] = 42;
  r.a.grid_h = 5; r.a.grid_w = 4; r.a.theta = 1e4;
  r.t[0] = {at, memory + 2048, 12 * 128, 128, 128, 100 * 128, 12};
  r.t[1] = {at, at, 4 * 128, 128, 4 * 128, 128, 4};
  r.n = 2;
  return r;
}

void rotate_refusals() {
  Ctx x;
  const float nan = std::numeric_limits<float>::quiet_NaN();
  refuses<Rot>(x.c, good_rotate(), {
      [](Rot &r) { r.n = 0; }, [](Rot &r) { r.n = 3; },
      [](Rot &r) { r.a.n_tokens = -1; },
      [](Rot &r) { r.a.head_dim = 0; }, [](Rot &r) { r.a.head_dim = 132; }, [](Rot &r) { r.a.head_dim = 264; },
      [](Rot &r) { r.a.x_type = 2; }, [](Rot &r) { r.a.out_type = -1; },
      [](Rot &r) { r.a.n_axes = 0; }, [](Rot &r) { r.a.n_axes = 5; }, [](Rot &r) { r.a.n_axes = 2; },
      [](Rot &r) { r.a.axis_dims[0] = 43; }, [](Rot &r) { r.a.axis_dims[1] = -2; },
      [](Rot &r) { r.a.axis_dims[0] = 60; }, [](Rot &r) { r.a.axis_dims[0] = 42; },
      [](Rot &r) { r.a.axis_dims[0] = r.a.axis_dims[1] = r.a.axis_dims[2] = 0; },
      [](Rot &r) { r.a.theta = 0; }, [](Rot &r) { r.a.theta = -1; }, [nan](Rot &r) { r.a.theta = nan; },
      [](Rot &r) { r.a.theta = INFINITY; },
      [](Rot &r) { r.a.grid_h = 0; }, [](Rot &r) { r.a.grid_w = -3; }, [](Rot &r) { r.a.frame0 = INT32_MAX; },
      [](Rot &r) { r.a.positions = (const int32_t *)(memory + 2); },
      [](Rot &r) { r.t[1].n_heads = 0; }, [](Rot &r) { r.t[0].n_heads = 70000; },
      [](Rot &r) { r.t[0].x = nullptr; }, [](Rot &r) { r.t[0].out = nullptr; },
      [](Rot &r) { r.t[0].x = memory + 8; }, [](Rot &r) { r.t[0].x_token = 12 * 128 + 4; },
      [](Rot &r) { r.t[0].x_head = -128; }, [](Rot &r) { r.t[0].out_head = 99 * 128; },
      [](Rot &r) { r.t[0].out_token = 0; },
      [](Rot &r) { r.t[1].out_token = 8 * 128; },                 // in place with other strides
      [](Rot &r) { r.a.out_type = HC_F32; },                      // in place with another type
  }, [&](const Rot &r) { return hc_rotate(x.c, &r.a, r.t, r.n, nullptr); });
  const Rot r = good_rotate();
  CHECK(hc_rotate(nullptr, &r.a, r.t, 2, nullptr) == HC_E_INVAL);
  CHECK(hc_rotate(x.c, nullptr, r.t, 2, nullptr) == HC_E_INVAL);
  CHECK(hc_rotate(x.c, &r.a, nullptr, 2, nullptr) == HC_E_INVAL);
  Rot none = r;
  none.a.n_tokens = 0;
  const int before = fake::launches;
  CHECK(hc_rotate(x.c, &none.a, none.t, 2, nullptr) == HC_OK && fake::launches == before);
  launch_result = hipErrorUnknown;
  CHECK(hc_rotate(x.c, &r.a, r.t, 2, nullptr) == HC_E_DEVICE);
  launch_result = hipSuccess;
  // turns per step: theta^(-2 j / m) / (2 pi), for each axis or for all pairs
  for (int joint = 0; joint < 2; ++joint) {
    Rot q = r;
    q.a.joint = joint;
    CHECK(hc_rotate(x.c, &q.a, q.t, 2, nullptr) == HC_OK);
    int pair = 0;
    for (int axis = 0; axis < 3; ++axis)
      for (int j = 0; j < q.a.axis_dims[axis] / 2; ++j, ++pair) {
        const double want = std::pow(1e4, joint ? -2.0 * pair / 128 : -2.0 * j / q.a.axis_dims[axis]) / (2 * M_PI);
        CHECK(std::fabs(rotated.turns[pair] - want) <= 1e-14 * want);
      }
    CHECK(rotated.axis_end[0] == 22 && rotated.axis_end[1] == 43 && rotated.axis_end[2] == 64);
  }
}

hc_packed_args good_packed() {
  hc_packed_args p{};
  p.q = p.k = p.v = at;
  p.out = memory + 2048;
  p.q_token = p.out_token = 8 * 64; p.k_token = p.v_token = 2 * 64;
  p.q_head = p.k_head = p.v_head = p.out_head = 64;
  p.n_tokens = 40; p.n_keys = 40; p.n_seqs = 3;
  p.n_heads = 8; p.n_kv_heads = 2; p.head_dim = 64; p.causal_block = 1;
  p.cu_q = iat;
  return p;
}

void packed_refusals() {
  Ctx x;
  using P = hc_packed_args;
  refuses<P>(x.c, good_packed(), {
      [](P &p) { p.n_tokens = -1; }, [](P &p) { p.n_keys = -1; }, [](P &p) { p.n_keys = 41; },
      [](P &p) { p.n_seqs = 0; }, [](P &p) { p.n_heads = 7; }, [](P &p) { p.n_kv_heads = 0; },
      [](P &p) { p.n_heads = 0; }, [](P &p) { p.head_dim = 96; }, [](P &p) { p.causal_block = -1; },
      [](P &p) { p.softmax_scale = -1; }, [](P &p) { p.softmax_scale = NAN; }, [](P &p) { p.softmax_scale = INFINITY; },
      [](P &p) { p.cu_q = nullptr; }, [](P &p) { p.cu_q = (const int32_t *)(memory + 1); },
      [](P &p) { p.cu_k = (const int32_t *)(memory + 2); },
      [](P &p) { p.q = nullptr; }, [](P &p) { p.k = nullptr; }, [](P &p) { p.v = memory + 8; },
      [](P &p) { p.out = nullptr; }, [](P &p) { p.k_token = 100; }, [](P &p) { p.v_head = -64; },
      [](P &p) { p.out_head = 56; }, [](P &p) { p.out_token = 0; },
      [](P &p) { p.n_tokens = p.n_keys = INT32_MAX; },
  }, [&](const P &p) { return hc_packed_attention(x.c, &p, nullptr); });
  P p = good_packed();
  CHECK(hc_packed_attention(nullptr, &p, nullptr) == HC_E_INVAL);
  CHECK(hc_packed_attention(x.c, nullptr, nullptr) == HC_E_INVAL);
  int64_t bytes = -1;
  CHECK(hc_packed_workspace(x.c, &p, nullptr) == HC_E_INVAL);
  CHECK(hc_packed_workspace(nullptr, &p, &bytes) == HC_E_INVAL);
  p.n_tokens = p.n_keys = 0;
  p.q = p.out = nullptr;
  const int before = fake::launches;
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK && fake::launches == before);
  // no keys: nothing to point at, and the outputs are written
  p = good_packed();
  p.n_keys = 0; p.k = p.v = nullptr; p.cu_k = iat;
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK && fake::launches == before + 1);
  // few rows over many keys: a workspace is asked for, and a smaller one is refused
  p = good_packed();
  p.cu_k = iat;
  p.n_keys = 300000;
  CHECK(hc_packed_workspace(x.c, &p, &bytes) == HC_OK && bytes > 0);
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_E_INVAL);
  p.workspace = memory + 1024;
  p.workspace_bytes = bytes - 1;
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_E_INVAL);
  p.workspace_bytes = bytes;
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK && merged && attended.n_split > 1);
  CHECK(bytes == (int64_t)attended.kv_heads * attended.tiles * (16 + attended.n_split * 128 * (64 + 2) * 4));
  p.workspace = memory + 1028;
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_E_INVAL);
}

void cache_refusals() {
  Ctx x;
  hc_qcache k{at, 3, 2, 64, 100};
  int64_t bytes = 0;
  CHECK(hc_qcache_bytes(&k, &bytes) == HC_OK && bytes == 3 * 2 * 2 * 64 * 2 * (32 + 2));
  CHECK(hc_qcache_bytes(nullptr, &bytes) == HC_E_INVAL && hc_qcache_bytes(&k, nullptr) == HC_E_INVAL);
  for (int i = 0; i < 6; ++i) {
    hc_qcache b = k;
    if (i == 0) b.n_seqs = 0;
    if (i == 1) b.n_heads = -1;
    if (i == 2) b.head_dim = 32;
    if (i == 3) b.capacity = 0;
    if (i == 4) b.capacity = INT32_MAX;
    if (i == 5) b.n_seqs = b.n_heads = b.capacity = INT32_MAX - 100;
    CHECK(hc_qcache_bytes(&b, &bytes) == HC_E_INVAL);
  }
  hc_qcache_rows r{at, memory + 2048, 128, 64, 128, 64, 9, iat, nullptr};
  using Rows = hc_qcache_rows;
  for (auto call : {hc_qcache_append, hc_qcache_read}) {
    refuses<Rows>(x.c, r, {
        [](Rows &r) { r.n_tokens = -1; }, [](Rows &r) { r.n_tokens = 10; }, [](Rows &r) { r.k = nullptr; },
        [](Rows &r) { r.v = memory + 4; }, [](Rows &r) { r.k_token = 12; }, [](Rows &r) { r.v_head = -8; },
        [](Rows &r) { r.start = nullptr; }, [](Rows &r) { r.start = (const int32_t *)(memory + 2); },
        [](Rows &r) { r.cu_seqlens = (const int32_t *)(memory + 2); },
        [](Rows &r) { r.n_tokens = INT32_MAX; r.cu_seqlens = iat; },
    }, [&](const Rows &r) { return call(x.c, &k, &r, nullptr); });
    hc_qcache bad = k;
    bad.data = nullptr;
    CHECK(call(x.c, &bad, &r, nullptr) == HC_E_INVAL);
    bad.data = memory + 8;
    CHECK(call(x.c, &bad, &r, nullptr) == HC_E_INVAL);
    CHECK(call(nullptr, &k, &r, nullptr) == HC_E_INVAL && call(x.c, nullptr, &r, nullptr) == HC_E_INVAL);
    CHECK(call(x.c, &k, nullptr, nullptr) == HC_E_INVAL);
    Rows none = r;
    none.n_tokens = 0;
    none.k = none.v = nullptr;
    const int before = fake::launches;
    CHECK(call(x.c, &k, &none, nullptr) == HC_OK && fake::launches == before);
  }
  Rows shared = r;            // one row for all tokens: fine to store, not to read into
  shared.k_token = 0;
  CHECK(hc_qcache_append(x.c, &k, &shared, nullptr) == HC_OK);
  CHECK(hc_qcache_read(x.c, &k, &shared, nullptr) == HC_E_INVAL);

  hc_qcache_attention_args a{};
  a.q = at; a.out = memory + 2048;
  a.q_token = a.out_token = 256; a.q_head = a.out_head = 64;
  a.n_tokens = 6; a.n_heads = 4; a.causal_block = 1; a.kv_len = iat;
  using A = hc_qcache_attention_args;
  refuses<A>(x.c, a, {
      [](A &a) { a.n_tokens = -1; }, [](A &a) { a.n_tokens = 7; }, [](A &a) { a.n_heads = 3; },
      [](A &a) { a.n_heads = 0; }, [](A &a) { a.causal_block = -2; }, [](A &a) { a.max_kv = -1; },
      [](A &a) { a.softmax_scale = -0.5f; }, [](A &a) { a.softmax_scale = NAN; }, [](A &a) { a.kv_len = nullptr; },
      [](A &a) { a.kv_len = (const int32_t *)(memory + 2); }, [](A &a) { a.cu_seqlens = (const int32_t *)(memory + 1); },
      [](A &a) { a.q = nullptr; }, [](A &a) { a.out = memory + 2; }, [](A &a) { a.q_token = 252; },
      [](A &a) { a.out_token = 128; }, [](A &a) { a.n_tokens = INT32_MAX; a.cu_seqlens = iat; },
  }, [&](const A &a) { return hc_qcache_attention(x.c, &k, &a, nullptr); });
  hc_qcache bad = k;
  bad.data = nullptr;
  CHECK(hc_qcache_attention(x.c, &bad, &a, nullptr) == HC_E_INVAL);
  CHECK(hc_qcache_workspace(x.c, &bad, &a, &bytes) == HC_OK && bytes == 0);    // no memory is looked at
  CHECK(hc_qcache_workspace(x.c, &k, &a, nullptr) == HC_E_INVAL);
  CHECK(hc_qcache_attention(nullptr, &k, &a, nullptr) == HC_E_INVAL);
  // a long cache is cut into ranges that need a workspace; the hint of a short one is not
  k.capacity = 100000;
  CHECK(hc_qcache_workspace(x.c, &k, &a, &bytes) == HC_OK && bytes > 0);
  CHECK(hc_qcache_attention(x.c, &k, &a, nullptr) == HC_E_INVAL);
  a.workspace = memory + 1024;
  a.workspace_bytes = bytes;
  CHECK(hc_qcache_attention(x.c, &k, &a, nullptr) == HC_OK && decoded && merged);
  a.max_kv = 50;
  CHECK(hc_qcache_workspace(x.c, &k, &a, &bytes) == HC_OK && bytes == 0);
}

// The units that sequences of any lengths need never exceed the room of the launch.
void unit_rooms() {
  Ctx x;
  uint32_t seed = 1;
  auto rnd = [&](int n) { seed = seed * 1664525u + 1013904223u; return (int)((seed >> 8) % (uint32_t)n); };
  hc_qcache k{at, 1, 1, 64, 4000};
  for (int round = 0; round < 2000; ++round) {
    const int n_seqs = 1 + rnd(40), group = 1 + rnd(9), longest = 1 + rnd(400);
    std::vector<int> len(n_seqs);
    int total = 0;
    for (int &n : len) total += n = rnd(3) ? rnd(longest) : 0;
    if (total == 0) total = len[0] = 1;
    auto needed = [&](int R) {
      int64_t u = 0;
      for (int n : len) u += (n * group + R - 1) / R;
      return u;
    };
    hc_packed_args p = good_packed();
    p.n_seqs = n_seqs; p.n_kv_heads = 1; p.n_heads = group; p.n_tokens = p.n_keys = total;
    p.q_token = p.out_token = 64 * group;
    p.workspace = at;
    p.workspace_bytes = INT64_MAX;
    CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK);
    CHECK(attended.tiles >= needed(kSeqRows));
    hc_qcache_attention_args a{};
    a.q = at; a.out = memory + 2048; a.q_token = a.out_token = 64 * group; a.q_head = a.out_head = 64;
    a.n_tokens = total; a.n_heads = group; a.kv_len = iat; a.cu_seqlens = iat;
    a.workspace = at;
    a.workspace_bytes = INT64_MAX;
    k.n_seqs = n_seqs;
    CHECK(hc_qcache_attention(x.c, &k, &a, nullptr) == HC_OK);
    CHECK(attended.tiles >= needed(decoded ? kDecodeRows : kSeqRows));
    // equal parts: exactly as many as they need
    p.n_tokens = p.n_keys = n_seqs * longest;
    p.cu_q = nullptr;
    CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK);
    CHECK(attended.tiles == n_seqs * ((longest * group + kSeqRows - 1) / kSeqRows));
  }
}

// A call runs on its context's device and leaves the caller's current.
void devices() {
  Ctx x;
  const Rot r = good_rotate();
  CHECK(hc_rotate(x.c, &r.a, r.t, 2, nullptr) == HC_OK);
  CHECK(device_in_launch == 0);
}

}  // namespace

int main(int argc, char **argv) {
  const std::string name = argc > 1 ? argv[1] : "";
  if (name == "rotate_refusals") rotate_refusals();
  else if (name == "packed_refusals") packed_refusals();
  else if (name == "cache_refusals") cache_refusals();
  else if (name == "unit_rooms") unit_rooms();
  else if (name == "devices") devices();
  else return 2;
  for (const std::string &f : fake::faults) std::fprintf(stderr, "%s\n", f.c_str());
  if (fails || !fake::faults.empty()) return 1;
  std::printf("%s: ok\n", name.c_str());
  return 0;
}
