// fused_dx.hip -- instances of the fused products, DX.
#include "fused_launch.h"

namespace gemm {
hipError_t launch_fused_dx(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s) { return launch_fused_op<FUSED_DX>(cfg, a, grid, s); }
}  // namespace gemm
