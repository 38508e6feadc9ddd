// mx_launch.h -- the launch functions of the block-scaled products, each in its own
// translation unit so that the library builds in parallel.
#pragma once

#include "mx_common.h"

namespace gemm {

// Each queues the kernel of configuration `cfg` (an index into kMxConfigs).
hipError_t launch_mx_fwd(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_mx_dx(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s);
hipError_t launch_mx_dw(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s);

// Rows of `used` bytes at any address and stride, copied to rows of `pitch` bytes (a multiple
// of 16) on 16-byte addresses, zeros behind each row: what the tile kernels load straight into
// LDS, 16 aligned bytes at a time.
struct MxCopy {
    const uint8_t *src;
    uint8_t *dst;
    int64_t stride, used, pitch, rows;     // rows 0: nothing to copy
};

template <typename K>
hipError_t launch_mx(K kernel, const MxArgs &a, dim3 grid, int threads, size_t lds, hipStream_t s) {
    hipLaunchKernelGGL(kernel, grid, dim3(unsigned(threads)), lds, s, a);
    return hipGetLastError();
}

}  // namespace gemm
