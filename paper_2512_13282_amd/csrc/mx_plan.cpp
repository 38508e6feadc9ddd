// mx_plan.cpp -- how the block-scaled products choose their kernel, tile and K slices (host).
#include "mx.h"

namespace gemm {

// Rows 0 and 1 are the decode kernel (at most 16 or 48 rows of A, A's K slice in 64 KiB of LDS), the
// rest are output tiles: mx_rows_kernel's where no waves are named, else mx_fwd_kernel's and
// mx_grad_kernel's.  The six figures of a tile are a least-squares fit of modelled_us to the logarithms of its own
// times (rows 1 to 11008, weights of 1024 x 1024 to 14336 x 4096, each in up to eight splits), and are to be fitted
// again where a kernel changes.  Checked over 150 other shapes, drawn over that range and a fifth of them odd, every
// plan of each timed (mx_force_plan): the chosen one takes 1.02 of the best one's time on geometric mean, within 3 % of
// it at 117 shapes, 1.33 at worst (25 x 4215 x 6533, forward: the decode kernel, for the copy that it saves).
const MxConfig kMxConfigs[] = {
    {MX_FWD, 16, 16, 8, 4, 0, 0, 0, 0, 0, 0, "mx_decode_16"},
    {MX_FWD, 48, 16, 8, 2, 0, 0, 0, 0, 0, 0, "mx_decode_48"},
    {MX_FWD, 32, 64, 8, 2, 2.17, 0.113, 0.308, 0.97, 4.21, 0.54, "mx_fwd_32x64_1x2x4"},
    {MX_FWD, 32, 128, 8, 1, 2.36, 0.167, 0.178, 0.83, 1.62, 0.12, "mx_fwd_32x128_1x4x2"},
    {MX_FWD, 64, 64, 8, 1, 3.01, 0.136, 0.153, 0.34, 3.46, 0.12, "mx_fwd_64x64_1x2x4"},
    {MX_FWD, 64, 128, 8, 1, 1.89, 0.226, 0.252, 0.74, 1.61, 0.37, "mx_fwd_64x128_1x4x2"},
    {MX_FWD, 128, 128, 8, 1, 1.93, 0.388, 0.414, 0.55, 1.44, 0.48, "mx_fwd_128x128_2x2x2"},
    {MX_FWD, 128, 128, 4, 2, 0.57, 0.516, 0.691, 1.44, 0.80, 0.48, "mx_fwd_128x128_2x2x1"},
    {MX_FWD, 128, 256, 8, 1, 0.09, 0.649, 0.708, 0.54, 0.89, 0.50, "mx_fwd_128x256_2x4x1"},
    {MX_FWD, 192, 256, 8, 1, 0.00, 0.982, 1.022, 0.00, 0.73, 0.41, "mx_fwd_192x256_2x4x1"},
    {MX_FWD, 256, 256, 8, 1, 0.00, 1.209, 1.266, 0.00, 0.81, 0.45, "mx_fwd_256x256_2x4x1"},
    {MX_DX, 16, 128, 8, 2, 0.24, 0.186, 0.321, 1.45, 2.55, 0.89, "mx_dx_16x128"},
    {MX_DX, 32, 128, 8, 1, 1.63, 0.208, 0.219, 0.32, 1.36, 0.69, "mx_dx_32x128"},
    {MX_DX, 48, 128, 8, 1, 2.31, 0.260, 0.253, 0.26, 1.14, 0.51, "mx_dx_48x128"},
    {MX_DX, 64, 128, 8, 1, 1.78, 0.442, 0.441, 0.79, 1.70, 0.41, "mx_dx_64x128_1x4x2"},
    {MX_DX, 64, 256, 8, 1, 0.18, 0.614, 0.598, 1.34, 0.99, 0.49, "mx_dx_64x256_1x8x1"},
    {MX_DX, 128, 128, 4, 2, 0.00, 0.677, 0.892, 1.69, 0.83, 0.43, "mx_dx_128x128_2x2x1"},
    {MX_DX, 128, 256, 8, 1, 0.00, 0.815, 0.808, 0.27, 0.85, 0.39, "mx_dx_128x256_2x4x1"},
    {MX_DX, 256, 256, 8, 1, 0.00, 1.222, 1.297, 0.00, 0.79, 0.37, "mx_dx_256x256_2x4x1"},
    {MX_DW, 32, 128, 8, 2, 1.12, 0.272, 0.483, 1.46, 0.97, 0.17, "mx_dw_32x128"},
    {MX_DW, 32, 64, 4, 3, 0.83, 0.344, 0.647, 1.97, 1.96, 0.21, "mx_dw_32x64_1x2x2"},
    {MX_DW, 64, 256, 8, 1, 0.00, 0.834, 0.908, 2.62, 1.06, 0.05, "mx_dw_64x256_1x8x1"},
    {MX_DW, 128, 128, 4, 2, 0.00, 0.861, 1.075, 1.79, 1.20, 0.09, "mx_dw_128x128_2x2x1"},
    {MX_DW, 128, 256, 8, 1, 0.56, 0.992, 0.974, 0.68, 0.95, 0.10, "mx_dw_128x256_2x4x1"},
    {MX_DW, 256, 256, 8, 1, 2.13, 1.372, 1.668, 0.00, 0.60, 0.10, "mx_dw_256x256_2x4x1"},
};
const int32_t kMxNumConfigs = sizeof(kMxConfigs) / sizeof(kMxConfigs[0]);

namespace {

constexpr int kCUs = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool evaluate(MxOp op, int64_t M, int64_t N, int64_t K, int32_t config, int32_t split, MxPlan *out) {
    if (config < 0 || config >= kMxNumConfigs || kMxConfigs[config].op != op) return false;
    const bool decode = config == kMxDecode || config == kMxDecode48;
    if (decode) {
        if (M > kMxConfigs[config].bm || K == 0) return false;
        const int64_t most = (65536 / M - 16) / 256 * 128;       // K of a slice that fits LDS
        const int64_t least = ceil_div(K, most);
        if (least > 4096) return false;
        if (split < least) split = int32_t(least);
    }
    const int64_t unit = decode ? 128 : 256;
    const int64_t chunk = K > 0 ? ceil_div(ceil_div(K, unit), split) * unit : unit;
    out->config = config;
    out->k_chunk = chunk;
    out->split_k = int32_t(K > 0 ? ceil_div(K, chunk) : 1);
    // A tile's partial sums are addressed with 32 bits, the decode kernel's slices are a grid dimension of
    // their own, and a dimension holds fewer than 2^32 threads.
    const MxConfig &c = kMxConfigs[config];
    const int64_t tiles = (decode ? 1 : ceil_div(M, c.bm)) * ceil_div(N, c.bn);
    const int64_t most = UINT32_MAX / (64 * c.waves) / (decode ? 1 : out->split_k);
    return out->split_k <= 65535 && int64_t(out->split_k) * c.bm * c.bn * 4 <= INT32_MAX && tiles <= most;
}

// Whether a configuration takes the operands, `copied_a` and `copied_b` bytes of which are not loadable: the
// decode kernel reads any rows, the rest can have theirs copied where a row is no longer than a stride may be.
bool holds(MxOp op, int64_t M, int64_t N, int64_t K, int64_t copied_a, int64_t copied_b, int32_t config) {
    if (config == kMxDecode || config == kMxDecode48) return true;
    return (copied_a == 0 || mx_a_row(op, M, K) <= kMxMostStride) && (copied_b == 0 || mx_b_row(op, N, K) <= kMxMostStride);
}

// Operands copied to aligned rows first: a launch and both ways through memory.
double copy_us(int64_t bytes) { return 3.5 + 2.0 * double(bytes) / 4.5e6; }

bool rows_dx(int32_t config) { return config >= 11 && config <= 13; }
bool rows_dw(int32_t config) { return config == 19; }

// What mx_rows_kernel loses to an A off 16-byte rows: its 16-byte pieces (DX), which every 128 columns of C
// read again, touch two lines each (130 x 4097 x 4095: 17.1 -> 29.4 us, 37 x 2049 x 2051: 6.9 -> 7.7);
// its dwords (DW) next to nothing (130 x 4097 x 4095: 22.0 -> 22.5).
double unaligned_us(int32_t config, int64_t M, int64_t N, int64_t K) {
    return rows_dx(config) ? 2.0 * double(M) * double(K) * double(ceil_div(N, 128)) / 2.9e6 : 0.0;
}

// Modelled microseconds of a plan, without the launch and what moves in any plan.
double modelled_us(MxOp op, int64_t M, int64_t N, int64_t K, const MxPlan &p, int64_t copied_b, int64_t copied_a) {
    const MxConfig &c = kMxConfigs[p.config];
    if (p.config == kMxDecode || p.config == kMxDecode48) {
        // W at the rate it streams at, A once for every 16 columns at the rate of the L2s.
        const double w = double(N) * double(K) / 2 / 5.0e6, a = double(ceil_div(N, 16)) * double(M) * double(K) * 2 / 8.5e6;
        return 0.7 + w + a + (p.split_k > 1 ? 1.0 : 0.0);
    }
    const double tiles = double(ceil_div(M, c.bm)) * double(ceil_div(N, c.bn)), groups = tiles * p.split_k;
    const double parts = double(p.k_chunk) / 64, slots = double(kCUs) * c.occupancy;
    const double alone = c.start_us + c.part_us * parts, shared = c.start_us + c.part_full_us * parts;
    const double rounds = double(int64_t(groups / slots)), rest = groups - rounds * slots;
    double t = rounds * (c.occupancy > 1 ? shared : alone);
    if (rest > 0) {
        const double per_cu = double(ceil_div(int64_t(rest), kCUs));     // on the fullest
        t += per_cu <= 1 ? alone : alone + (shared - alone) * (per_cu - 1) / (c.occupancy - 1);
    }
    const double tile = double(c.bm) * c.bn;
    t += c.store_us * tiles * tile * (op == MX_DW ? 4 : 2) / 1e6;
    if (p.split_k > 1) {
        // The last slice's sums, and every slice's partial sums out and back.
        const double rows = M < 8 ? 8 : M < c.bm ? double(M) : double(c.bm);
        t += c.sum_us + c.sum_slice_us * p.split_k * tile * 4 / 1e5 + groups * rows * c.bn * 8 / 4.5e6;
    }
    // No tile is faster than the operands' way out of memory, at the rate they stream at (124 MB for
    // 1 x 28672 x 8192: 31.7 us, where the decode kernel takes 28.0).
    const double moved = 2.0 * double(M) * double(K) + double(N) * double(K) * (op == MX_DW ? 1.03 : 0.53) +
                         double(M) * double(N) * (op == MX_DW ? 4 : 2);
    double copy = 0;
    if (copied_a > 0 && mx_direct_a(p.config, M, N, K)) {
        copy = unaligned_us(p.config, M, N, K);
        copied_a = 0;
    }
    if (copied_a + copied_b > 0) copy += copy_us(copied_a + copied_b);
    return (t > moved / 4.4e6 ? t : moved / 4.4e6) + copy;
}

}  // namespace

bool mx_direct_a(int32_t config, int64_t M, int64_t N, int64_t K) {
    if (config == kMxDecode || config == kMxDecode48) return true;
    if (rows_dw(config)) return M >= 2;                          // its dwords are two columns of A
    return rows_dx(config) && unaligned_us(config, M, N, K) < copy_us(2 * M * K);
}

bool mx_select(MxOp op, int64_t M, int64_t N, int64_t K, int64_t copied_a, int64_t copied_b, int32_t config, int32_t split,
               MxPlan *out) {
    if (config >= 0)
        return evaluate(op, M, N, K, config, split > 0 ? split : 1, out) && holds(op, M, N, K, copied_a, copied_b, config);
    static const int32_t kSplits[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32};
    double best = 0;
    bool found = false;
    for (int32_t c = 0; c < kMxNumConfigs; ++c) {
        if (kMxConfigs[c].op != op || !holds(op, M, N, K, copied_a, copied_b, c)) continue;
        int32_t seen = 0;
        for (const int32_t s : kSplits) {
            MxPlan p;
            if (!evaluate(op, M, N, K, c, split > 0 ? split : s, &p)) break;
            if (p.split_k == seen) continue;                     // the same slices again
            seen = p.split_k;
            // Partial sums stay a fraction of the memory.
            const double tiles = double(ceil_div(M, kMxConfigs[c].bm)) * double(ceil_div(N, kMxConfigs[c].bn));
            const double groups = tiles * p.split_k;
            if (split == 0 && p.split_k > 1 && kMxConfigs[c].bn > 16 && groups > 4 * kCUs) break;
            const double t = modelled_us(op, M, N, K, p, copied_b, copied_a);
            if (!found || t < best) {
                best = t;
                *out = p;
                found = true;
            }
            if (split > 0) break;
        }
    }
    return found;
}

}  // namespace gemm
