// mx_fwd.hip -- instances of the kernels over 4-bit weights, forward.
#include "kern_mx_decode.h"
#include "kern_mx_tile.h"
#include "mx_launch.h"

namespace gemm {

hipError_t launch_mx_fwd(int32_t cfg, const MxArgs &a, int64_t grid, hipStream_t s) {
    const dim3 g{unsigned(grid)};
    if (cfg == kMxDecode || cfg == kMxDecode48) {
        const size_t x = size_t(a.g.M) * size_t(a.g.k_chunk * 2 + 16), sums = size_t(kMxConfigs[cfg].bm / 16) * 8 * 1024 + 16;
        const dim3 d{unsigned(a.g.tiles_n), unsigned(a.g.split_k)};
        return cfg == kMxDecode ? launch_mx(mx_decode_kernel<1, 8, 2>, a, d, 512, x > sums ? x : sums, s)
                                : launch_mx(mx_decode_kernel<3, 8, 2>, a, d, 512, x > sums ? x : sums, s);
    }
    switch (cfg) {
        case 2: return launch_mx(mx_fwd_kernel<32, 64, 1, 2, 4, 2, 256, 3, 1024>, a, g, 512, 0, s);
        case 3: return launch_mx(mx_fwd_kernel<32, 128, 1, 4, 2, 2, 256, 3, 1024>, a, g, 512, 0, s);
        case 4: return launch_mx(mx_fwd_kernel<64, 64, 1, 2, 4, 2, 256, 3, 1024>, a, g, 512, 0, s);
        case 5: return launch_mx(mx_fwd_kernel<64, 128, 1, 4, 2, 2, 128, 3, 1024>, a, g, 512, 0, s);
        case 6: return launch_mx(mx_fwd_kernel<128, 128, 2, 2, 2, 2, 128, 3, 1024>, a, g, 512, 0, s);
        case 7: return launch_mx(mx_fwd_kernel<128, 128, 2, 2, 1, 2, 64, 3, 1024>, a, g, 256, 0, s);
        case 8: return launch_mx(mx_fwd_kernel<128, 256, 2, 4, 1, 2, 128, 3, 2048>, a, g, 512, 0, s);
        case 9: return launch_mx(mx_fwd_kernel<192, 256, 2, 4, 1, 2, 128, 2, 4096>, a, g, 512, 0, s);
        case 10: return launch_mx(mx_fwd_kernel<256, 256, 2, 4, 1, 2, 64, 3, 4096>, a, g, 512, 0, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace gemm
