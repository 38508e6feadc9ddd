// fused_dw.hip -- instances of the fused products, DW.
#include "fused_launch.h"

namespace gemm {
hipError_t launch_fused_dw(int32_t cfg, const FusedArgs &a, int64_t grid, hipStream_t s) { return launch_fused_op<FUSED_DW>(cfg, a, grid, s); }
}  // namespace gemm
