// Stand-ins for the device side of the feed-forward and adapter products, beside sanitize_stub.cpp: the CPU
// tests of the C ABI never reach a launch.
#include "../paper_2512_13282_amd/csrc/adapters.h"

namespace gemm {
int launch_fused(const FusedArgs &, FusedOp, const FusedPlan &, void *) { return LAUNCH_HIP_ERROR; }
int launch_gated_bwd(const GatedBwdArgs &, void *) { return LAUNCH_HIP_ERROR; }
int launch_adapters(const FusedArgs &, FusedOp, const FusedPlan &, const ShrinkArgs &, void *) { return LAUNCH_HIP_ERROR; }
int launch_adapters_dw(const AdapterDwArgs &, void *) { return LAUNCH_HIP_ERROR; }
}  // namespace gemm
