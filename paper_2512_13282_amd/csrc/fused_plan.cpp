// fused_plan.cpp -- how the fused products choose their tile and K slices (host).
#include "fused.h"

#include <math.h>

namespace gemm {

const FusedConfig kFusedConfigs[] = {
    {64, 128, 4, 2, 4096, 0, "fused_64x128_2x2"},
    {128, 256, 8, 1, 4096, 0, "fused_pingpong_128x256"},
    {192, 256, 8, 1, 4096, 0, "fused_pingpong_192x256"},
    {256, 256, 8, 1, 16, 0, "fused_pingpong_256x256"},
    {256, 256, 8, 1, 1, 192, "fused_pingpong_256x256_192"},
    {256, 256, 8, 1, 1, 128, "fused_pingpong_256x256_128"},
    {128, 128, 8, 1, 4096, 0, "fused_128x128_4x2"},
    {16, 16, 8, 2, 1, 0, "fused_decode_16"},
    {32, 16, 16, 1, 1, 0, "fused_decode_32"},
    {48, 16, 16, 1, 1, 0, "fused_decode_48"},
    {64, 16, 8, 2, 1, 0, "fused_decode_64"},
    {16, 16, 8, 1, 1, 0, "fused_stream_16"},
    {32, 16, 8, 1, 1, 0, "fused_stream_32"},
};
const int32_t kFusedNumConfigs = sizeof(kFusedConfigs) / sizeof(kFusedConfigs[0]);

namespace {

constexpr int kCUs = 256;
constexpr int32_t kFused128 = 1, kFused192 = 2, kFused256 = 3;     // rows of kFusedConfigs that the lower tiles' plans use too

// The model's figures: a least-squares fit of modelled_us to the logarithms of the times of every configuration and number
// of slices at 970 drawn shapes (rows 1 to 4096, widths of 64 to 14336, every operator, cold weights).  They are to be
// fitted again where a kernel changes.
struct FusedFigures {
    // Microseconds: a workgroup's start and end, a stage of 64 k of its tile alone on its compute unit and with the unit
    // full, a last slice's sum and its share per 100 KB of partial sums.
    double start_us, part_us, part_full_us, sum_us, sum_slice_us;
};
constexpr FusedFigures kFigures[] = {
    {1.341, 0.370, 0.619, 0.661, 0.000},
    {2.935, 0.673, 0.673, 1.871, 0.528},
    {4.314, 0.876, 0.876, 2.580, 0.411},
    {5.138, 1.084, 1.084, 2.438, 0.377},
    {}, {},                                          // with lower tiles: as the one without, and theirs
    {1.643, 0.509, 0.509, 1.746, 0.295},
};
// A stage's time by operator, over GATED's.
constexpr double kPart[FUSED_OPS][7] = {
    {1.000, 1.000, 1.000, 1.000, 0, 0, 1.000},
    {1.107, 1.167, 1.126, 1.133, 0, 0, 1.061},
    {0.970, 0.947, 0.889, 0.903, 0, 0, 0.962},
    {0.954, 0.988, 0.990, 1.062, 0, 0, 0.973},
    {0.936, 0.817, 0.828, 0.932, 0, 0, 0.929},
    {0.877, 0.824, 0.797, 0.831, 0, 0, 0.902},
};
constexpr double kStore[FUSED_OPS] = {0.312, 0.377, 0.393, 0.040, 0.344, 0.303};   // a megabyte of results (GRAD: and of G and U)
constexpr double kLaunch = 2.73, kRate = 4.85, kSlice = 0.51;                      // megabytes in a microsecond; each slice
constexpr double kEarly = 0.92;                                                    // GRAD's lower tiles that begin early
// The kernels for few rows: the start, a megabyte of weights and of A, 100 KB of both through one compute unit, 1000 k,
// a round of workgroups.
struct FewFigures { double start_us, weights_us, x_us, own_us, k_us, round_us; };
constexpr FewFigures kFew[] = {
    {3.809, 0.141, 0.108, 2.531, 0.000, 0.362}, {4.277, 0.188, 0.095, 2.733, 0.000, 0.006}, {3.256, 0.216, 0.075, 2.698, 0.213, 0.757},
    {2.049, 0.216, 0.090, 2.505, 0.605, 1.200}, {4.024, 0.137, 0.026, 0.843, 0.000, 1.069}, {4.220, 0.168, 0.026, 0.971, 0.000, 0.720},
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

double out_mb(FusedOp op, int32_t pairs, int64_t M, int64_t N) {
    static constexpr int kBytes[FUSED_OPS] = {6, 10, 2, 4, 2, 2};
    return double(kBytes[op]) * pairs * double(M) * double(N) / 1e6;
}

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

double moved_mb(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K) {
    const double m = double(M), n = double(N), k = double(K), two = op == FUSED_DX ? 2.0 : double(pairs);
    return (2.0 * two * m * k + 2.0 * (op == FUSED_GATED || op == FUSED_DX ? 2.0 : 1.0) * n * k) / 1e6 + out_mb(op, pairs, M, N);
}

// Rounds of `groups` workgroups with `stages` stages each.
double rounds_us(FusedOp op, int32_t config, double groups, double stages) {
    const FusedConfig &c = kFusedConfigs[config];
    const FusedFigures &f = kFigures[config];
    const double slots = double(kCUs) * c.occupancy, full = double(int64_t(groups / slots)), rest = groups - full * slots;
    const double part = kPart[op][config];
    const double alone = f.start_us + f.part_us * part * stages, shared = f.start_us + f.part_full_us * part * stages;
    double t = full * (c.occupancy > 1 ? shared : alone);
    if (rest > 0) {
        const double per_cu = double(ceil_div(int64_t(rest), kCUs));     // on the fullest
        t += per_cu <= 1 ? alone : alone + (shared - alone) * (per_cu - 1) / (c.occupancy - 1);
    }
    return t;
}

// Modelled microseconds of a plan, where `copied` bytes of the operands are not loadable.
double modelled_us(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K, const FusedPlan &p, int64_t copied) {
    const FusedConfig &c = kFusedConfigs[p.config];
    // Operands copied to aligned rows first: a launch and both ways through memory.
    const double copy = copied > 0 && !fused_any_address(p.config) ? 3.5 + 2.0 * double(copied) / 4.5e6 : 0.0;
    if (fused_few_rows(p.config)) {
        const FewFigures &f = kFew[p.config - kFusedDecode];
        const double rows = double(N) * (op == FUSED_GATED ? 2 : 1), groups = double(ceil_div(int64_t(rows), 16));
        const double tokens = double(M < c.bm ? M : c.bm), weights = 2.0 * rows * double(K) / 1e6, x = groups * tokens * double(K) * 2 / 1e6;
        const double per_cu = double(ceil_div(int64_t(groups), kCUs)), own = per_cu * 2.0 * (16 + tokens) * double(K) / 1e5;
        const double all = f.weights_us * weights + f.x_us * x, one = f.own_us * own;
        const double rounds = double(ceil_div(int64_t(groups), kCUs * (p.config < kFusedStream ? 2 : 1)));
        return f.start_us + (all > one ? all : one) + f.k_us * double(K) / 1e3 + f.round_us * rounds + copy;
    }
    const double stages = double(ceil_div(K, 64)) * (op == FUSED_DX ? 2 : 1), chunk = double(p.k_chunk) / 64;
    const int64_t tiles = ceil_div(M, c.bm) * pairs * ceil_div(N, op == FUSED_GATED ? c.bn / 2 : c.bn);
    const int32_t as = c.low > 0 ? kFused256 : p.config;
    double t = rounds_us(op, as, double(p.whole), stages) + kStore[op] * out_mb(op, pairs, M, N);
    if (c.low > 0) t += rounds_us(op, c.low == 192 ? kFused192 : kFused128, double(fused_tail(op, pairs, M, N, p).tiles), stages);
    if (p.split_k > 1) {
        // The slices, the last one's sum, and every slice's partial sums out and back.
        const FusedFigures &f = kFigures[as];
        const double groups = double(tiles - p.whole) * p.split_k, rows = M < 8 ? 8 : M < c.bm ? double(M) : double(c.bm);
        t += rounds_us(op, as, groups, chunk) + f.sum_us + kSlice * p.split_k + f.sum_slice_us * p.split_k * rows * c.bn * 4 / 1e5 + groups * rows * c.bn * 8 / 4.5e6;
    }
    const double memory = moved_mb(op, pairs, M, N, K) / kRate;
    if (op == FUSED_GRAD && c.low > 0) t *= kEarly;
    // Either hides the other in part only.
    return kLaunch + cbrt(t * t * t + memory * memory * memory) + copy;
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
        // Of two matrices the rows left are the second's: whole rounds have more than half of all tiles.
        const bool second = pairs == 2;
        t.row = (second ? p.tail_rows - per : p.tail_rows) * c.bm;
        t.tiles_m = ceil_div(M - t.row, c.low);
        t.half = second ? 0 : t.tiles_m;
        t.tiles_n = tn;
    }
    t.tiles = t.tiles_m * t.tiles_n;
    return t;
}

bool fused_has(FusedOp op, int32_t config) {
    if (op < 0 || op >= FUSED_OPS || config < 0 || config >= kFusedNumConfigs) return false;
    return !fused_few_rows(config) || op == FUSED_GATED || op == FUSED_ADAPT;
}

bool fused_select(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K, int64_t copied, int32_t config, int32_t split, FusedPlan *out) {
    if (config >= 0) return evaluate(op, pairs, M, N, K, config, split > 0 ? split : 1, out);
    static const int32_t kSplits[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32};
    double best = 0;
    bool found = false;
    for (int32_t c = 0; c < kFusedNumConfigs; ++c) {
        // Of the kernels for few rows at any address the first that holds them.
        if (c > kFusedDecode && fused_any_address(c) && M <= kFusedConfigs[c - 1].bm) continue;
        int32_t seen = 0;
        for (const int32_t s : kSplits) {
            FusedPlan p;
            if (!evaluate(op, pairs, M, N, K, c, split > 0 ? split : s, &p)) break;
            if (p.split_k == seen) continue;                     // the same slices again
            seen = p.split_k;
            const double t = modelled_us(op, pairs, M, N, K, p, copied);
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
