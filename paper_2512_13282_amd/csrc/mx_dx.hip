// mx_dx.hip -- instances of the gradient kernel, input gradients over 4-bit weights.
#include "kern_mx_tile.h"
#include "mx_launch.h"

namespace gemm {

hipError_t launch_mx_dx(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    switch (cfg) {
        case 6: return launch_mx(mx_grad_kernel<MX_DX, 32, 128, 1, 4, 1, 3, 2>, a, g, 256, 0, s);
        case 7: return launch_mx(mx_grad_kernel<MX_DX, 64, 128, 2, 2, 1, 3, 2>, a, g, 256, 0, s);
        case 8: return launch_mx(mx_grad_kernel<MX_DX, 128, 128, 2, 2, 1, 2, 2>, a, g, 256, 0, s);
        case 9: return launch_mx(mx_grad_kernel<MX_DX, 256, 256, 2, 4, 1, 2, 2>, a, g, 512, 0, s);
        case 29: return launch_mx(mx_grad_kernel<MX_DX, 32,64,1,2,4,2,3>, a, g, 512, 0, s);
        case 30: return launch_mx(mx_grad_kernel<MX_DX, 32,64,1,2,2,4,3>, a, g, 256, 0, s);
        case 31: return launch_mx(mx_grad_kernel<MX_DX, 32,128,1,4,2,2,3>, a, g, 512, 0, s);
        case 32: return launch_mx(mx_grad_kernel<MX_DX, 64,64,1,2,2,2,3>, a, g, 256, 0, s);
        case 33: return launch_mx(mx_grad_kernel<MX_DX, 64,128,1,4,2,2,3>, a, g, 512, 0, s);
        case 34: return launch_mx(mx_grad_kernel<MX_DX, 64,128,2,2,2,2,3>, a, g, 512, 0, s);
        case 35: return launch_mx(mx_grad_kernel<MX_DX, 64,128,2,2,1,3,3>, a, g, 256, 0, s);
        case 36: return launch_mx(mx_grad_kernel<MX_DX, 128,64,2,1,1,2,3>, a, g, 128, 0, s);
        case 37: return launch_mx(mx_grad_kernel<MX_DX, 128,128,2,2,1,2,3>, a, g, 256, 0, s);
        case 38: return launch_mx(mx_grad_kernel<MX_DX, 64,256,1,8,1,2,3>, a, g, 512, 0, s);
        case 39: return launch_mx(mx_grad_kernel<MX_DX, 128,256,2,4,1,2,3>, a, g, 512, 0, s);
        case 40: return launch_mx(mx_grad_kernel<MX_DX, 128,256,2,4,1,4,2>, a, g, 512, 0, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace gemm
