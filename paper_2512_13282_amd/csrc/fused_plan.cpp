// fused_plan.cpp -- how the fused products choose their tile and K slices (host).
#include "fused.h"

namespace gemm {

const FusedConfig kFusedConfigs[] = {
    {64, 128, 4, 2, 4096, 0, "fused_64x128_2x2"},
    {128, 256, 8, 1, 4096, 0, "fused_pingpong_128x256"},
    {192, 256, 8, 1, 4096, 0, "fused_pingpong_192x256"},
    {256, 256, 8, 1, 16, 0, "fused_pingpong_256x256"},
    {256, 256, 8, 1, 1, 192, "fused_pingpong_256x256_192"},
    {256, 256, 8, 1, 1, 128, "fused_pingpong_256x256_128"},
    {16, 16, 8, 2, 1, 0, "fused_decode_16"},
    {32, 16, 8, 2, 1, 0, "fused_decode_32"},
    {48, 16, 8, 2, 1, 0, "fused_decode_48"},
    {64, 16, 8, 2, 1, 0, "fused_decode_64"},
    {16, 16, 8, 1, 1, 0, "fused_stream_16"},
    {32, 16, 8, 1, 1, 0, "fused_stream_32"},
};
const int32_t kFusedNumConfigs = sizeof(kFusedConfigs) / sizeof(kFusedConfigs[0]);

namespace {

constexpr int kCUs = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool evaluate(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K, int32_t config, int32_t split, FusedPlan *out) {
    if (config < 0 || config >= kFusedNumConfigs || !fused_has(op, config)) return false;
    const FusedConfig &c = kFusedConfigs[config];
    if (split > c.most_slices || (fused_few_rows(config) && M > c.bm)) return false;
    const int64_t stages = ceil_div(K, 64) * (op == FUSED_DX ? 2 : 1);
    const int64_t tm = ceil_div(M, c.bm) * pairs, tn = ceil_div(N, op == FUSED_GATED ? c.bn / 2 : c.bn), tiles = tm * tn;
    if (tiles > INT32_MAX) return false;
    // Tiles that fill whole rounds of the compute units keep all of K.
    const int64_t slots = int64_t(kCUs) * c.occupancy, rest = tiles % slots;
    const int64_t chunk = stages > 0 && rest > 0 ? ceil_div(stages, split) : stages > 0 ? stages : 1;
    out->config = config;
    out->k_chunk = 64 * chunk;
    out->split_k = int32_t(stages > 0 ? ceil_div(stages, chunk) : 1);
    out->tail_rows = out->tail_cols = 0;
    const int64_t sliced = out->split_k > 1 ? rest : 0;
    int64_t groups = tiles - sliced + sliced * out->split_k;
    out->whole = int32_t(tiles - sliced);
    if (c.low > 0) {
        // The tile columns or rows that fill whole rounds, whichever wastes less; lower tiles over the others.
        const int64_t full = tiles - rest, cols = full / tm, rows = full / tn;
        if (full == 0 || rest == 0) return false;
        if (cols * tm >= rows * tn) out->tail_cols = int32_t(cols);
        else out->tail_rows = int32_t(rows);
        out->whole = int32_t(out->tail_cols > 0 ? cols * tm : rows * tn);
        groups = out->whole + fused_tail(op, pairs, M, N, *out).tiles;
    }
    // A tile's partial sums are addressed with 32 bits, and a grid holds fewer than 2^32 threads.
    return int64_t(out->split_k) * c.bm * c.bn * 4 <= INT32_MAX && groups <= UINT32_MAX / (64 * c.waves);
}

// Modelled microseconds of a plan, without the launch.
double modelled_us(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t, const FusedPlan &p) {
    const FusedConfig &c = kFusedConfigs[p.config];
    const double tiles = double(ceil_div(M, c.bm)) * pairs * double(ceil_div(N, op == FUSED_GATED ? c.bn / 2 : c.bn));
    const double groups = tiles * p.split_k, rounds = double(int64_t(groups / (kCUs * c.occupancy)) + 1);
    return rounds * (2.0 + 0.4 * double(p.k_chunk) / 64) + (p.split_k > 1 ? 3.0 + 0.2 * p.split_k : 0.0);
}

}  // namespace

FusedTail fused_tail(FusedOp op, int32_t pairs, int64_t M, int64_t N, const FusedPlan &p) {
    const FusedConfig &c = kFusedConfigs[p.config];
    const int64_t width = op == FUSED_GATED ? c.bn / 2 : c.bn, per = ceil_div(M, c.bm), tn = ceil_div(N, width);
    FusedTail t{};
    if (p.tail_cols > 0) {
        t.col = p.tail_cols * width;
        t.half = ceil_div(M, c.low);
        t.tiles_m = t.half * pairs;
        t.tiles_n = tn - p.tail_cols;
    } else {
        const bool second = p.tail_rows >= per;                  // the rows left are all the second matrix's
        t.row = (second ? p.tail_rows - per : p.tail_rows) * c.bm;
        const int64_t left = ceil_div(M - t.row, c.low);
        t.half = second ? 0 : left;
        t.tiles_m = second ? left : left + (pairs == 2 ? ceil_div(M, c.low) : 0);
        t.tiles_n = tn;
    }
    t.tiles = t.tiles_m * t.tiles_n;
    return t;
}

bool fused_has(FusedOp op, int32_t config) {
    if (op < 0 || op >= FUSED_OPS || config < 0 || config >= kFusedNumConfigs) return false;
    return !fused_few_rows(config) || op == FUSED_GATED || op == FUSED_ADAPT;
}

bool fused_select(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K, int32_t config, int32_t split, FusedPlan *out) {
    if (config >= 0) return evaluate(op, pairs, M, N, K, config, split > 0 ? split : 1, out);
    static const int32_t kSplits[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32};
    double best = 0;
    bool found = false;
    for (int32_t c = 0; c < kFusedNumConfigs; ++c) {
        int32_t seen = 0;
        for (const int32_t s : kSplits) {
            FusedPlan p;
            if (!evaluate(op, pairs, M, N, K, c, split > 0 ? split : s, &p)) break;
            if (p.split_k == seen) continue;                     // the same slices again
            seen = p.split_k;
            const double t = modelled_us(op, pairs, M, N, K, p);
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
