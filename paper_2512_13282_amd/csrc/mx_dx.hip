// mx_dx.hip -- instances of the gradient kernels, input gradients over 4-bit weights.
#include "kern_mx_rows.h"
#include "kern_mx_tile.h"
#include "mx_launch.h"

namespace gemm {

hipError_t launch_mx_dx(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    switch (cfg) {
        case 11: return launch_mx(mx_rows_kernel<MX_DX, 1, 8, 2, 4>, a, g, 512, 0, s);
        case 12: return launch_mx(mx_rows_kernel<MX_DX, 2, 8, 2, 2>, a, g, 512, 0, s);
        case 13: return launch_mx(mx_rows_kernel<MX_DX, 3, 8, 2, 2>, a, g, 512, 0, s);
        case 14: return launch_mx(mx_grad_kernel<MX_DX, 64, 128, 1, 4, 2, 2>, a, g, 512, 0, s);
        case 15: return launch_mx(mx_grad_kernel<MX_DX, 64, 256, 1, 8, 1, 2>, a, g, 512, 0, s);
        case 16: return launch_mx(mx_grad_kernel<MX_DX, 128, 128, 2, 2, 1, 2>, a, g, 256, 0, s);
        case 17: return launch_mx(mx_grad_kernel<MX_DX, 128, 256, 2, 4, 1, 2>, a, g, 512, 0, s);
        case 18: return launch_mx(mx_grad_kernel<MX_DX, 256, 256, 2, 4, 1, 2>, a, g, 512, 0, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace gemm
