// More checks of the entry points beside the routed attention (hc_ops.cpp) on the CPU: calls at the
// ends of their ranges.  As ops_check.cpp, against the HIP runtime of fake_hip.h, but with
// devices that are told apart.  One check per run, by name.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <functional>
#include <string>

#include <hip/hip_runtime.h>

#define hipSetDevice ignored_set_device       // (fake_hip.h's looks at no device)
#include "fake_hip.h"
#undef hipSetDevice
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

int device_now = 0, device_in_launch = -1;      // the calling thread's
hipError_t launch_result = hipSuccess;
RotateArgs rotated;
SeqArgs attended;
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
hipError_t launch_rotate(const RotateArgs &a, int, int, bool, hipStream_t) { rotated = a; return launched(); }
hipError_t launch_qcache_append(const QCacheArgs &, hipStream_t) { return launched(); }
hipError_t launch_qcache_read(const QCacheArgs &, hipStream_t) { return launched(); }
hipError_t launch_seq(const SeqArgs &a, int, hipStream_t) { attended = a; return launched(); }
hipError_t launch_decode(const SeqArgs &a, int, hipStream_t) { attended = a; return launched(); }
hipError_t launch_seq_merge(const SeqArgs &, int, int, hipStream_t) { return launched(); }
}  // namespace hc

namespace {

struct Ctx {
  hc_ctx *c = nullptr;
  explicit Ctx(int device = 0) {
    hc_config cfg;
    hc_config_default(&cfg);
    CHECK(hc_create(&cfg, device, &c) == HC_OK);
  }
  ~Ctx() { hc_destroy(c); }
};

alignas(16) char memory[4096];
const int32_t *const iat = (const int32_t *)memory;

hc_packed_args good_packed() {
  hc_packed_args p{};
  p.q = p.k = p.v = memory;
  p.out = memory + 2048;
  p.q_token = p.out_token = 64; p.k_token = p.v_token = 64;
  p.q_head = p.k_head = p.v_head = p.out_head = 64;
  p.n_tokens = 1; p.n_keys = 1; p.n_seqs = 1;
  p.n_heads = 1; p.n_kv_heads = 1; p.head_dim = 64;
  p.cu_k = iat;
  return p;
}

// A call is refused with a message and without a launch.
void refused(hc_ctx *c, const std::function<hc_status()> &call, const char *word) {
  const int before = fake::launches;
  CHECK(call() == HC_E_INVAL);
  CHECK(fake::launches == before);
  if (!std::strstr(hc_last_error(c), word)) {
    std::fprintf(stderr, "message '%s' lacks '%s'\n", hc_last_error(c), word);
    ++fails;
  }
}

// The kernels count key tiles in 32 bits: more keys than those hold are refused, though keys of
// stride 0 need no memory for them; the most that they hold run.
void key_counts() {
  Ctx x;
  hc_packed_args p = good_packed();
  p.k_token = p.v_token = 0;
  int64_t bytes = 0;
  for (int n : {INT32_MAX, INT32_MAX - kSeqKeys + 1}) {
    p.n_keys = n;
    refused(x.c, [&] { return hc_packed_attention(x.c, &p, nullptr); }, "keys");
    refused(x.c, [&] { return hc_packed_workspace(x.c, &p, &bytes); }, "keys");
  }
  p.n_keys = INT32_MAX - kSeqKeys;
  CHECK(hc_packed_workspace(x.c, &p, &bytes) == HC_OK);
  p.workspace = memory;
  p.workspace_bytes = bytes;
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK && attended.n_keys == p.n_keys);
}

// The scale is used times log2(e): what leaves the floats there is refused as if it were infinite.
void large_scales() {
  Ctx x;
  hc_packed_args p = good_packed();
  hc_qcache k{memory, 1, 1, 64, 64};
  hc_qcache_attention_args a{};
  a.q = memory; a.out = memory + 2048;
  a.q_token = a.out_token = a.q_head = a.out_head = 64;
  a.n_tokens = 1; a.n_heads = 1; a.kv_len = iat;
  for (float scale : {3e38f, 2.4e38f}) {
    p.softmax_scale = a.softmax_scale = scale;
    refused(x.c, [&] { return hc_packed_attention(x.c, &p, nullptr); }, "softmax_scale");
    refused(x.c, [&] { return hc_qcache_attention(x.c, &k, &a, nullptr); }, "softmax_scale");
  }
  for (float scale : {2.3e38f, 1e-38f, 0.f}) {
    p.softmax_scale = a.softmax_scale = scale;
    CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_OK && std::isfinite(attended.scale_log2));
    CHECK(hc_qcache_attention(x.c, &k, &a, nullptr) == HC_OK && std::isfinite(attended.scale_log2));
  }
}

// A theta so small that an angle of a far position leaves the doubles is refused.
void small_thetas() {
  Ctx x;
  hc_rotate_args a{};
  a.n_tokens = 1; a.head_dim = 64; a.n_axes = 1; a.axis_dims[0] = 64; a.positions = iat;
  hc_rotate_tensor t{memory, memory + 2048, 64, 64, 64, 64, 1};
  for (double theta : {5e-324, 1e-315, 1e-310}) {
    a.theta = theta;
    refused(x.c, [&] { return hc_rotate(x.c, &a, &t, 1, nullptr); }, "theta");
  }
  for (double theta : {1e-307, 1e-3, 1.0, 1e300}) {   // (1e-307: 4.1e296 turns a step, 8.7e305 at 2^31)
    a.theta = theta;
    CHECK(hc_rotate(x.c, &a, &t, 1, nullptr) == HC_OK);
    for (int i = 0; i < 32; ++i) CHECK(std::isfinite(rotated.turns[i] * -0x1p31));
  }
}

// Every call launches on its context's device and leaves the caller's current, whatever the launch returns
// and however the call ends.
void call_devices() {
  Ctx x;
  hc_rotate_args r{};
  r.n_tokens = 1; r.head_dim = 64; r.n_axes = 1; r.axis_dims[0] = 64; r.positions = iat; r.theta = 1e4;
  const hc_rotate_tensor t{memory, memory + 2048, 64, 64, 64, 64, 1};
  hc_qcache k{memory, 1, 1, 64, 64};
  hc_qcache_rows rows{memory, memory + 2048, 64, 64, 64, 64, 1, iat, nullptr};
  hc_qcache_attention_args a{};
  a.q = memory; a.out = memory + 2048;
  a.q_token = a.out_token = a.q_head = a.out_head = 64;
  a.n_tokens = 1; a.n_heads = 1; a.kv_len = iat;
  hc_packed_args p = good_packed(), many = good_packed();      // whole, and in key ranges
  many.n_keys = 100000;
  many.k_token = many.v_token = 0;
  CHECK(hc_packed_workspace(x.c, &many, &many.workspace_bytes) == HC_OK && many.workspace_bytes > 0);
  many.workspace = memory;
  const std::function<hc_status()> calls[] = {
      [&] { return hc_rotate(x.c, &r, &t, 1, nullptr); },
      [&] { return hc_packed_attention(x.c, &p, nullptr); },
      [&] { return hc_packed_attention(x.c, &many, nullptr); },
      [&] { return hc_qcache_append(x.c, &k, &rows, nullptr); },
      [&] { return hc_qcache_read(x.c, &k, &rows, nullptr); },
      [&] { return hc_qcache_attention(x.c, &k, &a, nullptr); },
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
  device_now = 1;
  p.head_dim = 96;                 // a refused call
  CHECK(hc_packed_attention(x.c, &p, nullptr) == HC_E_INVAL && device_now == 1);
  device_now = 0;
}

}  // namespace

int main(int argc, char **argv) {
  const std::string name = argc > 1 ? argv[1] : "";
  if (name == "key_counts") key_counts();
  else if (name == "large_scales") large_scales();
  else if (name == "small_thetas") small_thetas();
  else if (name == "call_devices") call_devices();
  else return 2;
  for (const std::string &f : fake::faults) std::fprintf(stderr, "%s\n", f.c_str());
  if (fails || !fake::faults.empty()) return 1;
  std::printf("%s: ok\n", name.c_str());
  return 0;
}
