// fused_launch.h -- the launch functions of the fused products, each in its own translation unit so
// that the library builds in parallel.
#pragma once

#include "kern_fused_pingpong.h"

namespace gemm {

// Each queues the kernel of configuration `cfg` (an index into kFusedConfigs).
hipError_t launch_fused_gated(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_grad(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_dx(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_dw(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_adapt(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_adapt_dx(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);

template <int OP>
hipError_t launch_fused_op(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    switch (cfg) {
        case 0: hipLaunchKernelGGL((fused_tile_kernel<OP, 64, 128, 2, 2, 2, 3>), g, dim3(256), 0, s, a); break;
        case 1: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 1, 1>), g, dim3(512), 0, s, a); break;
        case 2: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 2, 1>), g, dim3(512), 0, s, a); break;
        case 3: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 2, 2>), g, dim3(512), 0, s, a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace gemm
