// Launchers that do nothing, for the CPU test of the plans of ress_layer.h's kernels (layer_plan.cpp,
// linked with them as it is), and the plans by C names. A call that passes every check ends in a
// launcher here, whose error it returns.
#include "layer_internal.h"

namespace ress {
hipError_t launch_norm(const NormParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_norm_bwd(const NormBwdParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_rope(const RopeParams &, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_window(const WindowParams &, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_window_bwd(const WindowBwdParams &, int, hipStream_t) { return hipErrorInvalidValue; }
hipError_t launch_decode(const DecodeParams &, hipStream_t) { return hipErrorInvalidValue; }
}  // namespace ress

extern "C" {
void plan_window(const ress_window_shape *s, int *out)
{
    const ress::WindowPlan p = ress::window_plan(s);
    out[0] = p.groups, out[1] = p.splits;
}
void plan_window_bwd(const ress_window_shape *s, int *out)
{
    const ress::WindowBwdPlan p = ress::window_bwd_plan(s);
    out[0] = p.groups, out[1] = p.sink_blocks, out[2] = p.sink_slices, out[3] = p.slices, out[4] = p.items;
}
int plan_joined(int sink_blocks, int sink_slices, int slices, int blocks, int *first)
{
    return ress::window_bwd_joined({1, sink_blocks, sink_slices, slices, 0}, blocks, *first);
}
int plan_decode(const ress_decode_shape *s) { return ress::decode_splits(s); }
int plan_norm_bwd(int64_t rows) { return ress::norm_bwd_parts(rows); }
}
