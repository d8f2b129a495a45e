// Gradients of the attention with a window, 64-dim heads.
#include "hc_window_grad.h"

namespace hc {

hipError_t launch_grad64(const GradArgs &a, hipStream_t s) { return launch<64>(a, s); }

}  // namespace hc
