// fused_gated.hip -- instances of the fused products, GATED.
#include "fused_launch.h"

namespace gemm {
hipError_t launch_fused_gated(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s) { return launch_fused_op<FUSED_GATED>(cfg, a, grid, s); }
}  // namespace gemm
