// Launchers and plans that do nothing, linked in place of the kernels of ress_layer.h when its C
// ABI layer is built with host sanitizers for the CPU tests: no call there reaches a launcher.
#include "layer_internal.h"

namespace ress {
int norm_bwd_parts(int64_t rows) { return (int)(rows < 1 ? 1 : rows < 512 ? rows : 512); }
WindowPlan window_plan(const ress_window_shape *) { return {4, 2}; }
WindowBwdPlan window_bwd_plan(const ress_window_shape *s) { return {1, 1, 2, 1, (s->n_k + 127) / 128 + 1}; }
int decode_splits(const ress_decode_shape *) { return 3; }
hipError_t launch_norm(const NormParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_norm_bwd(const NormBwdParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_rope(const RopeParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_window(const WindowParams &, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_window_bwd(const WindowBwdParams &, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_decode(const DecodeParams &, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace ress

extern "C" int divided(int n, int d) { return ress::divider(d)(n); }
