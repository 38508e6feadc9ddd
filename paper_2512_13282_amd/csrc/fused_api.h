// fused_api.h -- what ffn_api.cpp and adapters_api.cpp share (host side).
#pragma once

#include <stdint.h>

#include <atomic>

#include "../../include/gemm_mi355x.h"
#include "fused.h"
#include "region.h"

namespace gemm {

constexpr int64_t kFusedMostSize = INT32_MAX - 4096;      // 32-bit indices, up to the end of a tile or a stage

// What a test or a benchmark forces: a configuration and a number of slices for each operator.
struct FusedForced {
    std::atomic<int32_t> config{-1}, split{0};
};

inline int fused_status(int launched) {
    switch (launched) {
        case LAUNCH_OK: return GEMM_OK;
        case LAUNCH_NO_MEMORY: return GEMM_ERR_NO_MEMORY;
        default: return GEMM_ERR_HIP;
    }
}

// Bytes of an operand that the tile kernels have copied first, and whether they can where they have to.
inline int64_t fused_copied(const void *p, int64_t ld, int64_t rows, int64_t cols, bool along_k) {
    return rows == 0 || cols == 0 || fused_loadable(p, ld, along_k, cols) ? 0 : 2 * rows * cols;
}
inline bool fused_copyable(const void *p, int64_t ld, int64_t rows, int64_t cols, bool along_k) {
    return rows == 0 || cols == 0 || fused_loadable(p, ld, along_k, cols) || (2 * cols + 15) / 16 * 16 <= kFusedMostStride;
}

// The plans of this thread's latest calls: choosing one evaluates dozens.
struct FusedCachedPlan {
    int64_t M, N, K, copied;                               // M = 0: empty
    int32_t op, pairs;
    FusedPlan plan;
};

inline int fused_plan_for(FusedOp op, int32_t pairs, int64_t M, int64_t N, int64_t K, int64_t copied, const FusedForced &forced, FusedPlan *plan) {
    if (M > kFusedMostSize || N > kFusedMostSize || K > kFusedMostSize) return GEMM_ERR_UNSUPPORTED;
    const int32_t config = forced.config, split = forced.split;
    if (config >= 0 || split > 0) return fused_select(op, pairs, M, N, K, copied, config, split, plan) ? GEMM_OK : GEMM_ERR_UNSUPPORTED;
    static thread_local FusedCachedPlan plans[64];
    const uint64_t h = (uint64_t(M) * 0x9E3779B97F4A7C15u ^ uint64_t(N) * 0xC2B2AE3D27D4EB4Fu ^ uint64_t(K) * 0x165667B19E3779F9u) + uint64_t(op);
    FusedCachedPlan &c = plans[(h ^ (h >> 32)) % 64];
    if (c.M != M || c.N != N || c.K != K || c.copied != copied || c.op != op || c.pairs != pairs) {
        FusedPlan p;
        if (!fused_select(op, pairs, M, N, K, copied, -1, 0, &p)) return GEMM_ERR_UNSUPPORTED;
        c = FusedCachedPlan{M, N, K, copied, op, pairs, p};
    }
    *plan = c.plan;
    return GEMM_OK;
}

}  // namespace gemm
