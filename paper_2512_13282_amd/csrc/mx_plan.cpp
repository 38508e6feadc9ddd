// mx_plan.cpp -- how the block-scaled products choose their kernel, tile and K slices (host).
#include "mx.h"

namespace gemm {

// Rows 0 and 1 are the decode kernels (at most kMxDecodeRows rows of A), the rest output tiles.
const MxConfig kMxConfigs[] = {
    {MX_FWD, 16, 16, 4, 8, "mx_decode_16_w4"},
    {MX_FWD, 16, 16, 8, 4, "mx_decode_16_w8"},
    {MX_FWD, 32, 64, 8, 2, "mx_fwd_32x64_1x2x4"},
    {MX_FWD, 32, 128, 8, 1, "mx_fwd_32x128_1x4x2"},
    {MX_FWD, 64, 64, 8, 1, "mx_fwd_64x64_1x2x4"},
    {MX_FWD, 64, 128, 8, 1, "mx_fwd_64x128_1x4x2"},
    {MX_FWD, 128, 128, 8, 1, "mx_fwd_128x128_2x2x2"},
    {MX_FWD, 128, 128, 4, 2, "mx_fwd_128x128_2x2x1"},
    {MX_FWD, 128, 256, 8, 1, "mx_fwd_128x256_2x4x1"},
    {MX_FWD, 192, 256, 8, 1, "mx_fwd_192x256_2x4x1"},
    {MX_FWD, 256, 256, 8, 1, "mx_fwd_256x256_2x4x1"},
    {MX_DX, 32, 64, 8, 1, "mx_dx_32x64_1x2x4"},
    {MX_DX, 32, 64, 4, 3, "mx_dx_32x64_1x2x2"},
    {MX_DX, 64, 64, 4, 2, "mx_dx_64x64_1x2x2"},
    {MX_DX, 64, 128, 8, 1, "mx_dx_64x128_1x4x2"},
    {MX_DX, 64, 256, 8, 1, "mx_dx_64x256_1x8x1"},
    {MX_DX, 128, 128, 4, 2, "mx_dx_128x128_2x2x1"},
    {MX_DX, 128, 256, 8, 1, "mx_dx_128x256_2x4x1"},
    {MX_DX, 256, 256, 8, 1, "mx_dx_256x256_2x4x1"},
    {MX_DW, 32, 64, 8, 1, "mx_dw_32x64_1x2x4"},
    {MX_DW, 32, 64, 4, 3, "mx_dw_32x64_1x2x2"},
    {MX_DW, 64, 64, 4, 2, "mx_dw_64x64_1x2x2"},
    {MX_DW, 64, 128, 8, 1, "mx_dw_64x128_1x4x2"},
    {MX_DW, 64, 256, 8, 1, "mx_dw_64x256_1x8x1"},
    {MX_DW, 128, 128, 4, 2, "mx_dw_128x128_2x2x1"},
    {MX_DW, 128, 256, 8, 1, "mx_dw_128x256_2x4x1"},
    {MX_DW, 256, 256, 8, 1, "mx_dw_256x256_2x4x1"},
};
const int32_t kMxNumConfigs = sizeof(kMxConfigs) / sizeof(kMxConfigs[0]);

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

static bool evaluate(MxOp op, int64_t M, int64_t K, int32_t config, int32_t split, MxPlan *out) {
    if (config < 0 || config >= kMxNumConfigs || kMxConfigs[config].op != op) return false;
    const bool decode = config < 2;
    if (decode) {
        // A's slice has to fit 64 KiB of LDS.
        if (M > 16 || K == 0) return false;
        const int64_t most = (65536 / M - 16) / 256 * 128;
        const int64_t least = ceil_div(K, most);
        if (split < least) split = int32_t(least);
    }
    const int64_t unit = decode ? 128 : 256;
    const int64_t chunk = K > 0 ? ceil_div(ceil_div(K, unit), split) * unit : unit;
    out->config = config;
    out->k_chunk = chunk;
    out->split_k = int32_t(K > 0 ? ceil_div(K, chunk) : 1);
    return true;
}

bool mx_select(MxOp op, int64_t M, int64_t N, int64_t K, int32_t config, int32_t split, MxPlan *out) {
    if (config >= 0) return evaluate(op, M, K, config, split > 0 ? split : 1, out);
    if (op == MX_FWD && M <= 4 && K > 0) return evaluate(op, M, K, N >= 8192 ? 0 : 1, 1, out);
    for (int c = 0; c < kMxNumConfigs; ++c)
        if (kMxConfigs[c].op == op && kMxConfigs[c].bm >= 32 && (kMxConfigs[c].bm >= M || kMxConfigs[c].bm >= 64)) return evaluate(op, M, K, c, split > 0 ? split : 1, out);
    return false;
}

}  // namespace gemm
