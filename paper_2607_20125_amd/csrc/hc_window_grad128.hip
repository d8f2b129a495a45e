// Gradients of the attention with a window, 128-dim heads.
#include "hc_window_grad.h"

namespace hc {

hipError_t launch_grad128(const GradArgs &a, hipStream_t s) { return launch<128>(a, s); }

}  // namespace hc
