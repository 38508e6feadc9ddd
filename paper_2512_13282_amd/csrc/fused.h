// fused.h -- interface between the feed-forward and adapter entry points (ffn_api.cpp,
// adapters_api.cpp) and their kernels.  Pure C++: no HIP types, as launch.h.
#pragma once

#include <stdint.h>

#include "launch.h"

namespace gemm {

// The products that do more than C = A . B, all over bf16 operands with fp32 sums.
enum FusedOp : int32_t {
    FUSED_GATED = 0,     // act(A . B^T) * (A . B2^T), B and B2 N x K
    FUSED_GRAD = 1,      // D = A . B, then D U act'(G), D act(G) and act(G) U; B K x N
    FUSED_DX = 2,        // A . B + A2 . B2, B and B2 K x N
    FUSED_DW = 3,        // A^T . B, and A2^T . B where there is an A2; A and A2 K x M, B K x N
    FUSED_ADAPT = 4,     // A . B^T + h Q_i^T, B N x K, Q_i N x r
    FUSED_ADAPT_DX = 5,  // A . B + h Q_i, B K x N, Q_i r x N
    FUSED_OPS = 6
};

struct FusedArgs {
    KernelArgs g;                    // first operands and result, sizes, tiles, slices, workspace
    const void *A2, *B2;
    int64_t lda2, ldb2;
    void *C2, *C3;                   // GATED: G and U (or null); GRAD: dU and H (H or null); DW: the second result
    int64_t ldc2, ldc3;
    const void *G, *U;               // GRAD
    int64_t ldg, ldu;
    int32_t act;                     // FFN_* of ffn_mi355x.h
    int32_t pairs;                   // DW: 1 or 2 matrices A
    int32_t whole;                   // workgroups with a tile and all of K, ahead of the rest
    int32_t early;                   // of the lower tiles, that many come after the first 128 workgroups
    int32_t half;                    // DW: tile rows of the first matrix
    struct Tail {                    // the lower tiles, where the plan has some: from row `row` and column `col` on
        int64_t row, col;
        int32_t tiles_m, tiles_n, half;
    } tail;
    // ADAPT: row t's h is the sum over `planes` of h[plane][t][0 .. r), its adapter index[t] in [0, n), any other
    // value for none; adapter i's matrix starts sq elements after the one before it, rows ldq apart.
    const float *h;
    int64_t h_plane;                 // elements from plane to plane; rows are r apart
    int32_t planes, n, r;
    const int32_t *index;
    const void *Q;
    int64_t ldq, sq;
};

// How a product runs: a row of kFusedConfigs and the number of K slices.
struct FusedPlan {
    int32_t config;
    int32_t split_k;                 // slices of each tile after the first `whole`
    int32_t whole;
    int32_t tail_rows, tail_cols;    // else the tile rows and columns that tiles of the whole height have, where lower
                                     // ones have the rest (0, 0: none)
    int64_t k_chunk;                 // K of a slice, a multiple of 64 (DX: of both products' K one after the other)
};

struct FusedConfig {
    int32_t bm, bn;                  // output tile; GATED: bn / 2 columns of each product
    int32_t waves;                   // per workgroup
    int32_t occupancy;               // workgroups that a compute unit holds
    int32_t most_slices;
    int32_t low;                     // rows of the lower tiles of a last round, 0: none
    const char *name;
};
extern const FusedConfig kFusedConfigs[];
extern const int32_t kFusedNumConfigs;

// The region that a plan's lower tiles cover: from a row (of the matrix that the others leave off in) or a column on.
struct FusedTail {
    int64_t row, col, tiles_m, tiles_n, tiles, half;         // half: tile rows of the first matrix
};
FusedTail fused_tail(FusedOp op, int32_t pairs, int64_t M, int64_t N, const FusedPlan &p);

// The kernels for few rows of A, by rows: the one that takes its operands as they lie, and the one for operands on
// 16-byte rows.
constexpr int32_t kFusedDecode = 7, kFusedStream = 11;
inline bool fused_few_rows(int32_t config) { return config >= kFusedDecode; }
inline bool fused_any_address(int32_t config) { return config >= kFusedDecode && config < kFusedStream; }

// Whether a configuration is built for an operator.
bool fused_has(FusedOp op, int32_t config);

// The plan for a product, where `copied` bytes of its operands are not loadable (below); config >= 0 and split > 0 say which
// one to take instead.  False where none (the one named does not) takes the sizes.
bool fused_select(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K, int64_t copied, int32_t config, int32_t split, FusedPlan *out);

// The tile kernels load 16 aligned bytes at a time straight into LDS, at 32-bit offsets within a
// tile: an operand whose rows lie otherwise is copied first.  Along the sum a row is whole pieces,
// for what lies behind its end would be part of the sum.
constexpr int64_t kFusedMostStride = int64_t(1) << 22;
inline bool fused_loadable(const void *p, int64_t ld, bool along_k, int64_t cols) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * 2 % 16 == 0 && ld * 2 <= kFusedMostStride &&
           (!along_k || cols % 8 == 0);
}

// dG and dU of M x N from dH, G and U.
struct GatedBwdArgs {
    int64_t M, N;
    const void *dH, *G, *U;
    void *dG, *dU;
    int64_t lddh, ldg, ldu, lddg, lddu;
    int32_t act;
};

// Each queues its kernels on `stream` (a hipStream_t) and returns a LAUNCH_* value.
int launch_gated_bwd(const GatedBwdArgs &a, void *stream);
int launch_fused(const FusedArgs &a, FusedOp op, const FusedPlan &plan, void *stream);

}  // namespace gemm
