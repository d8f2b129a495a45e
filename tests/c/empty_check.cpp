// Calls of the rotation and of the norm without tokens (hc_ops.cpp, hc_window.cpp) on the CPU: hc_rotate looks at
// its arguments as it does with tokens, the norm takes the NULL that an empty tensor of positions has.  Compiled with
// hc_runtime.cpp against the HIP runtime of fake_hip.h.
#include <functional>

#include "fake_hip.h"
#include "hc_ops.h"
#include "hc_window.h"
#include "headcast.h"

using namespace hc;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
}
namespace {
hipError_t launched() { ++fake::launches; return hipSuccess; }
}
namespace hc {
hipError_t launch_rotate(const RotateArgs &, int, int, bool, hipStream_t) { return launched(); }
hipError_t launch_qcache_append(const QCacheArgs &, hipStream_t) { return launched(); }
hipError_t launch_qcache_read(const QCacheArgs &, hipStream_t) { return launched(); }
hipError_t launch_seq(const SeqArgs &, int, hipStream_t) { return launched(); }
hipError_t launch_decode(const SeqArgs &, int, hipStream_t) { return launched(); }
hipError_t launch_seq_merge(const SeqArgs &, int, int, hipStream_t) { return launched(); }
hipError_t launch_norm(const NormArgs &, int, int, bool, hipStream_t) { return launched(); }
hipError_t launch_norm_backward(const NormArgs &, int, int, bool, hipStream_t) { return launched(); }
hipError_t launch_paged_append(const PagedRowsArgs &, hipStream_t) { return launched(); }
hipError_t launch_window(const SeqArgs &, int, hipStream_t) { return launched(); }
hipError_t launch_paged_decode(const SeqArgs &, int, hipStream_t) { return launched(); }
hipError_t launch_grad64(const GradArgs &, hipStream_t) { return launched(); }
hipError_t launch_grad128(const GradArgs &, hipStream_t) { return launched(); }
}  // namespace hc

int main() {
  int fails = 0;
  hc_config cfg;
  hc_config_default(&cfg);
  hc_ctx *c = nullptr;
  if (hc_create(&cfg, 0, &c) != HC_OK) return 2;
  hc_rotate_args good{};
  good.head_dim = 128;
  good.x_type = good.out_type = HC_BF16;
  good.n_axes = 3;
  good.axis_dims[0] = 44;
  good.axis_dims[1] = good.axis_dims[2] = 42;
  good.grid_h = 4;
  good.grid_w = 5;
  good.theta = 10000;
  hc_rotate_tensor t{};
  t.n_heads = 2;
  hc_norm_tensor nt{};
  nt.n_heads = 2;
  const std::function<void(hc_rotate_args &)> bad[] = {
      [](hc_rotate_args &a) { a.grid_h = 0; }, [](hc_rotate_args &a) { a.grid_w = -1; },
      [](hc_rotate_args &a) { a.frame0 = INT32_MAX; },
      [](hc_rotate_args &a) { a.n_axes = 2; a.axis_dims[0] = a.axis_dims[1] = 64; a.axis_dims[2] = 0; }};
  auto expect = [&](bool ok, const char *what, int i) {
    if (ok) return;
    std::fprintf(stderr, "%s %d: message '%s'\n", what, i, hc_last_error(c));
    ++fails;
  };
  const int before = fake::launches;
  expect(hc_rotate(c, &good, &t, 1, nullptr) == HC_OK, "rotate", -1);
  int i = 0;
  for (const auto &change : bad) {
    hc_rotate_args a = good;
    change(a);
    expect(hc_rotate(c, &a, &t, 1, nullptr) == HC_E_INVAL, "rotate", i);
    const hc_norm_args n{a, HC_F32, 1e-6f};
    expect(hc_norm_rotate(c, &n, &nt, 1, nullptr) == HC_OK, "norm", i);
    ++i;
  }
  expect(fake::launches == before, "launches", fake::launches - before);
  hc_destroy(c);
  if (!fails) std::printf("ok\n");
  return fails != 0;
}
