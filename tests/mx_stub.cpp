// Stand-ins for the device side of the block-scaled products, beside sanitize_stub.cpp: the CPU
// tests of the C ABI never reach a launch.
#include "../paper_2512_13282_amd/csrc/mx.h"

namespace gemm {
int launch_mx_pack(const MxMatrixArgs &, int, void *) { return LAUNCH_HIP_ERROR; }
int launch_mx_unpack(const MxMatrixArgs &, int, void *) { return LAUNCH_HIP_ERROR; }
int launch_mx_gemm(const MxArgs &, MxOp, const MxPlan &, void *) { return LAUNCH_HIP_ERROR; }
}  // namespace gemm
