// mx_plan.cpp -- how the block-scaled products choose their kernel, tile and K slices (host).
#include "mx.h"

namespace gemm {

// Rows 0 and 1 are the decode kernels (at most kMxDecodeRows rows of A), the rest output tiles.
const MxConfig kMxConfigs[] = {
    {MX_FWD, 16, 16, 4, 8, "mx_decode_16_w4"},
    {MX_FWD, 16, 16, 8, 4, "mx_decode_16_w8"},
    {MX_FWD, 32, 128, 4, 2, "mx_fwd_32x128"},
    {MX_FWD, 64, 128, 4, 2, "mx_fwd_64x128"},
    {MX_FWD, 128, 128, 4, 2, "mx_fwd_128x128"},
    {MX_FWD, 256, 256, 8, 1, "mx_fwd_256x256"},
    {MX_DX, 32, 128, 4, 3, "mx_dx_32x128"},
    {MX_DX, 64, 128, 4, 2, "mx_dx_64x128"},
    {MX_DX, 128, 128, 4, 2, "mx_dx_128x128"},
    {MX_DX, 256, 256, 8, 1, "mx_dx_256x256"},
    {MX_DW, 32, 128, 4, 3, "mx_dw_32x128"},
    {MX_DW, 64, 128, 4, 2, "mx_dw_64x128"},
    {MX_DW, 128, 128, 4, 2, "mx_dw_128x128"},
    {MX_DW, 256, 256, 8, 1, "mx_dw_256x256"},
    {MX_FWD, 32, 128, 8, 2, "mx_T14_32x128_1x4x2_w2_k128_n3"},
    {MX_FWD, 32, 128, 8, 2, "mx_T15_32x128_1x4x2_w2_k128_n4"},
    {MX_FWD, 32, 128, 8, 1, "mx_T16_32x128_1x4x2_w2_k256_n3"},
    {MX_FWD, 32, 128, 16, 1, "mx_T17_32x128_1x4x4_w4_k256_n2"},
    {MX_FWD, 32, 128, 8, 2, "mx_T18_32x128_1x4x2_w4_k128_n2"},
    {MX_FWD, 64, 128, 8, 1, "mx_T19_64x128_1x4x2_w2_k128_n3"},
    {MX_FWD, 64, 128, 8, 1, "mx_T20_64x128_2x2x2_w2_k128_n3"},
    {MX_FWD, 128, 256, 8, 1, "mx_T21_128x256_2x4x1_w2_k64_n3"},
    {MX_FWD, 128, 256, 8, 2, "mx_T22_128x256_2x4x1_w4_k64_n2"},
    {MX_FWD, 64, 128, 8, 1, "mx_T23_64x128_1x4x2_w2_k256_n2"},
    {MX_FWD, 32, 128, 8, 1, "mx_T24_32x128_1x2x4_w2_k256_n3"},
    {MX_FWD, 64, 64, 8, 1, "mx_T25_64x64_1x2x4_w2_k256_n3"},
    {MX_FWD, 32, 64, 8, 1, "mx_T26_32x64_1x2x4_w2_k256_n3"},
    {MX_FWD, 64, 64, 8, 1, "mx_T27_64x64_2x2x2_w2_k256_n2"},
    {MX_FWD, 128, 128, 8, 1, "mx_T28_128x128_2x2x2_w2_k128_n3"},
    {MX_DX, 32, 64, 8, 1, "mx_T29_32x64_1x2x4_w2_a3"},
    {MX_DX, 32, 64, 4, 2, "mx_T30_32x64_1x2x2_w4_a3"},
    {MX_DX, 32, 128, 8, 2, "mx_T31_32x128_1x4x2_w2_a3"},
    {MX_DX, 64, 64, 4, 2, "mx_T32_64x64_1x2x2_w2_a3"},
    {MX_DX, 64, 128, 8, 1, "mx_T33_64x128_1x4x2_w2_a3"},
    {MX_DX, 64, 128, 8, 1, "mx_T34_64x128_2x2x2_w2_a3"},
    {MX_DX, 64, 128, 4, 2, "mx_T35_64x128_2x2x1_w3_a3"},
    {MX_DX, 128, 64, 2, 2, "mx_T36_128x64_2x1x1_w2_a3"},
    {MX_DX, 128, 128, 4, 1, "mx_T37_128x128_2x2x1_w2_a3"},
    {MX_DX, 64, 256, 8, 1, "mx_T38_64x256_1x8x1_w2_a3"},
    {MX_DX, 128, 256, 8, 1, "mx_T39_128x256_2x4x1_w2_a3"},
    {MX_DX, 128, 256, 8, 1, "mx_T40_128x256_2x4x1_w4_a2"},
    {MX_DW, 32, 64, 8, 1, "mx_T41_32x64_1x2x4_w2_a3"},
    {MX_DW, 32, 64, 4, 2, "mx_T42_32x64_1x2x2_w4_a3"},
    {MX_DW, 32, 128, 8, 2, "mx_T43_32x128_1x4x2_w2_a3"},
    {MX_DW, 64, 64, 4, 2, "mx_T44_64x64_1x2x2_w2_a3"},
    {MX_DW, 64, 128, 8, 1, "mx_T45_64x128_1x4x2_w2_a3"},
    {MX_DW, 64, 128, 8, 1, "mx_T46_64x128_2x2x2_w2_a3"},
    {MX_DW, 64, 128, 4, 2, "mx_T47_64x128_2x2x1_w3_a3"},
    {MX_DW, 128, 64, 2, 2, "mx_T48_128x64_2x1x1_w2_a3"},
    {MX_DW, 128, 128, 4, 1, "mx_T49_128x128_2x2x1_w2_a3"},
    {MX_DW, 64, 256, 8, 1, "mx_T50_64x256_1x8x1_w2_a3"},
    {MX_DW, 128, 256, 8, 1, "mx_T51_128x256_2x4x1_w2_a3"},
    {MX_DW, 128, 256, 8, 1, "mx_T52_128x256_2x4x1_w4_a2"},
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
    const int first = op == MX_FWD ? 2 : op == MX_DX ? 6 : 10;
    const int at = M <= 32 ? 0 : M <= 64 ? 1 : M <= 512 || N <= 1024 ? 2 : 3;
    const MxConfig &c = kMxConfigs[first + at];
    const int64_t tiles = ceil_div(M, c.bm) * ceil_div(N, c.bn);
    int64_t s = 256 * c.occupancy / tiles;
    if (s > ceil_div(K, 512)) s = ceil_div(K, 512);
    return evaluate(op, M, K, first + at, int32_t(split > 0 ? split : s < 1 ? 1 : s > 32 ? 32 : s), out);
}

}  // namespace gemm
