// fused_grad.hip -- instances of the fused products, GRAD.
#include "fused_launch.h"

namespace gemm {
hipError_t launch_fused_grad(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s) { return launch_fused_op<FUSED_GRAD>(cfg, a, grid, s); }
}  // namespace gemm
