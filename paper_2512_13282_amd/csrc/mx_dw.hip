// mx_dw.hip -- instances of the gradient kernels, weight gradients over 8-bit checkpoints.
#include "kern_mx_rows.h"
#include "kern_mx_tile.h"
#include "mx_launch.h"

namespace gemm {

hipError_t launch_mx_dw(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    switch (cfg) {
        case 19: return launch_mx(mx_rows_kernel<MX_DW, 2, 8, 1, 4>, a, g, 512, 0, s);
        case 20: return launch_mx(mx_grad_kernel<MX_DW, 32, 64, 1, 2, 2, 4>, a, g, 256, 0, s);
        case 21: return launch_mx(mx_grad_kernel<MX_DW, 64, 256, 1, 8, 1, 2>, a, g, 512, 0, s);
        case 22: return launch_mx(mx_grad_kernel<MX_DW, 128, 128, 2, 2, 1, 2>, a, g, 256, 0, s);
        case 23: return launch_mx(mx_grad_kernel<MX_DW, 128, 256, 2, 4, 1, 2>, a, g, 512, 0, s);
        case 24: return launch_mx(mx_grad_kernel<MX_DW, 256, 256, 2, 4, 1, 2>, a, g, 512, 0, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace gemm
