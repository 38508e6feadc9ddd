// adapters.h -- interface between adapters_api.cpp and the kernels.  Pure C++: no HIP types, as launch.h.
#pragma once

#include <stdint.h>

#include "fused.h"

namespace gemm {

// h = s_i P Q_i over tokens' rows P (M x L): Q_i is r x L (QT) or L x r.
struct ShrinkArgs {
    const void *P;
    int64_t ldp, M, L;
    const void *Q;
    int64_t ldq, sq;
    const float *scale;          // or null
    const int32_t *index;
    int32_t n, r;
    bool qt;
    float *h;                    // the caller's (M x r), or null: the workspace's
    float *out;                  // where the kernel writes: planes of M x r
    uint32_t *counters;          // of the token blocks and rank groups: the slices are added up into h; or null
    int64_t plane;
    int32_t slices;              // of L, a plane each, at most 8
    int32_t blocks, groups;      // of tokens and of ranks
    int64_t chunk;               // L of a slice, a multiple of 32
    int32_t parts;               // workgroups that share the adapters of a block
};

struct AdapterDwArgs {
    int64_t M;
    int32_t n, r;
    const int32_t *index;
    struct Side {
        const void *z;           // M x cols
        int64_t ldz, cols;
        const float *h;          // M x r
        void *out;               // n matrices, r x cols (side 0) or cols x r (side 1)
        int64_t ld, stride;
        int32_t blocks;          // of columns
    } side[2];
    int32_t bf16_out;
};

constexpr int64_t kAdaptersMostRank = 1024;

// Each queues its kernels on `stream` (a hipStream_t) and returns a LAUNCH_* value.  launch_adapters: the adapters'
// first product, then `a` (ADAPT or ADAPT_DX) with it; rank 0 and no adapters are the product with W alone.
int launch_adapters(const FusedArgs &a, FusedOp op, const FusedPlan &plan, const ShrinkArgs &s, void *stream);
int launch_adapters_dw(const AdapterDwArgs &a, void *stream);

}  // namespace gemm
