// fused_launch.h -- the launch functions of the fused products, each in its own translation unit so
// that the library builds in parallel.
#pragma once

#include "kern_fused_decode.h"
#include "kern_fused_pingpong.h"

namespace gemm {

// Each queues the kernel of configuration `cfg` (an index into kFusedConfigs).
hipError_t launch_fused_gated(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_grad(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_dx(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_dw(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_adapt(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_fused_adapt_dx(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s);

template <int OP, int MT, int KW, int U>
void launch_decode(const FusedArgs &a, dim3 grid, bool odd, hipStream_t s) {
    if (odd) hipLaunchKernelGGL((fused_decode_kernel<OP, MT, KW, U, true>), grid, dim3(64 * KW), 0, s, a);
    else hipLaunchKernelGGL((fused_decode_kernel<OP, MT, KW, U, false>), grid, dim3(64 * KW), 0, s, a);
}

template <int OP>
hipError_t launch_fused_op(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    switch (cfg) {
        case 0: hipLaunchKernelGGL((fused_tile_kernel<OP, 64, 128, 2, 2, 2, 3>), g, dim3(256), 0, s, a); break;
        case 1: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 1, 1, 0, 0>), g, dim3(512), 0, s, a); break;
        case 2: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 2, 1, 0, 0>), g, dim3(512), 0, s, a); break;
        case 3: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 2, 2, 0, 0>), g, dim3(512), 0, s, a); break;
        case 4: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 2, 2, 2, 1>), g, dim3(512), 0, s, a); break;
        case 5: hipLaunchKernelGGL((fused_pingpong_kernel<OP, 2, 2, 1, 1>), g, dim3(512), 0, s, a); break;
        case 6: hipLaunchKernelGGL((fused_tile_kernel<OP, 128, 128, 4, 2, 2, 3>), g, dim3(512), 0, s, a); break;
        default:
            if constexpr (OP == FUSED_GATED || OP == FUSED_ADAPT) {
                // Whether any 16 bytes of a row may lie off a dword.
                const auto off = [](const void *p, int64_t ld, int64_t rows) { return reinterpret_cast<uintptr_t>(p) % 4 != 0 || (ld % 2 != 0 && rows > 1); };
                const bool odd = off(a.g.A, a.g.lda, a.g.M) || off(a.g.B, a.g.ldb, a.g.N) || (OP == FUSED_GATED && off(a.B2, a.ldb2, a.g.N));
                // Sixteen waves shorten each one's way through K, but a compute unit holds one such workgroup: GATED has
                // twice as many (37 x 2051 x 2049: 257, 20.7 against 25.6 us; ADAPT 129, 21.1 against 19.8).
                constexpr int FEW = OP == FUSED_ADAPT ? 16 : 8;
                if (cfg == kFusedDecode + 0) launch_decode<OP, 1, 8, 4>(a, g, odd, s);
                else if (cfg == kFusedDecode + 1) launch_decode<OP, 2, FEW, 2>(a, g, odd, s);
                else if (cfg == kFusedDecode + 2) launch_decode<OP, 3, FEW, 2>(a, g, odd, s);
                else if (cfg == kFusedDecode + 3) launch_decode<OP, 4, 8, 2>(a, g, odd, s);
                else if (cfg == kFusedStream) hipLaunchKernelGGL((fused_stream_kernel<OP, 1, 8, 4>), g, dim3(512), 0, s, a);
                else if (cfg == kFusedStream + 1) hipLaunchKernelGGL((fused_stream_kernel<OP, 2, 8, 2>), g, dim3(512), 0, s, a);
                else return hipErrorInvalidValue;
                break;
            } else {
                return hipErrorInvalidValue;
            }
    }
    return hipGetLastError();
}

}  // namespace gemm
