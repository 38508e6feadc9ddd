// mx_dw.hip -- instances of the gradient kernel, weight gradients over 8-bit checkpoints.
#include "kern_mx_tile.h"
#include "mx_launch.h"

namespace gemm {

hipError_t launch_mx_dw(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    switch (cfg) {
        case 10: return launch_mx(mx_grad_kernel<MX_DW, 32, 128, 1, 4, 1, 3, 2>, a, g, 256, 0, s);
        case 11: return launch_mx(mx_grad_kernel<MX_DW, 64, 128, 2, 2, 1, 3, 2>, a, g, 256, 0, s);
        case 12: return launch_mx(mx_grad_kernel<MX_DW, 128, 128, 2, 2, 1, 2, 2>, a, g, 256, 0, s);
        case 13: return launch_mx(mx_grad_kernel<MX_DW, 256, 256, 2, 4, 1, 2, 2>, a, g, 512, 0, s);
        case 41: return launch_mx(mx_grad_kernel<MX_DW, 32,64,1,2,4,2,3>, a, g, 512, 0, s);
        case 42: return launch_mx(mx_grad_kernel<MX_DW, 32,64,1,2,2,4,3>, a, g, 256, 0, s);
        case 43: return launch_mx(mx_grad_kernel<MX_DW, 32,128,1,4,2,2,3>, a, g, 512, 0, s);
        case 44: return launch_mx(mx_grad_kernel<MX_DW, 64,64,1,2,2,2,3>, a, g, 256, 0, s);
        case 45: return launch_mx(mx_grad_kernel<MX_DW, 64,128,1,4,2,2,3>, a, g, 512, 0, s);
        case 46: return launch_mx(mx_grad_kernel<MX_DW, 64,128,2,2,2,2,3>, a, g, 512, 0, s);
        case 47: return launch_mx(mx_grad_kernel<MX_DW, 64,128,2,2,1,3,3>, a, g, 256, 0, s);
        case 48: return launch_mx(mx_grad_kernel<MX_DW, 128,64,2,1,1,2,3>, a, g, 128, 0, s);
        case 49: return launch_mx(mx_grad_kernel<MX_DW, 128,128,2,2,1,2,3>, a, g, 256, 0, s);
        case 50: return launch_mx(mx_grad_kernel<MX_DW, 64,256,1,8,1,2,3>, a, g, 512, 0, s);
        case 51: return launch_mx(mx_grad_kernel<MX_DW, 128,256,2,4,1,2,3>, a, g, 512, 0, s);
        case 52: return launch_mx(mx_grad_kernel<MX_DW, 128,256,2,4,1,4,2>, a, g, 512, 0, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace gemm
