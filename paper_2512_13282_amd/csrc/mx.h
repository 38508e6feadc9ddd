// mx.h -- interface between the block-scaled entry points (mx_api.cpp) and their kernels.
// Pure C++: no HIP types, as launch.h.
#pragma once

#include <stdint.h>

#include "launch.h"

namespace gemm {

constexpr int kMxBlock = 32;     // elements of a row that share one scale byte

// The products: what B is and along which index its blocks lie.
enum MxOp : int32_t {
    MX_FWD = 0,   // C = A . B^T, B 4-bit N x K (blocks along K)
    MX_DX = 1,    // C = A . B,   B 4-bit K x N (blocks along N)
    MX_DW = 2     // C = A^T . B, A bf16 K x M, B 8-bit K x N (blocks along N)
};

struct MxArgs {
    KernelArgs g;              // A, C and the sizes; B: the codes, ldb: their row stride in bytes
    const uint8_t *scales;
    int64_t ld_scales;         // row stride in bytes
};

struct MxMatrixArgs {          // packing and unpacking
    int64_t rows, cols;
    void *x;                   // bf16, read or written
    int64_t ldx;               // elements
    void *codes;
    int64_t ldq;               // bytes
    uint8_t *scales;
    int64_t ld_scales;         // bytes
};

// How a product runs: a row of kMxConfigs and the number of K slices.
struct MxPlan {
    int32_t config;
    int32_t split_k;
    int64_t k_chunk;           // K of a slice, a multiple of 256 (the decode kernel's: of 128)
};

struct MxConfig {
    MxOp op;
    int32_t bm, bn;            // output tile
    int32_t waves;             // per workgroup
    int32_t occupancy;         // workgroups a compute unit holds
    // Fitted microseconds: a workgroup's start and its end, 64 k of its K alone on its compute
    // unit and with the unit full, a split's last slice and its share per 100 KB of partial
    // sums, and 1 MB of results.
    double start_us, part_us, part_full_us, sum_us, sum_slice_us, store_us;
    const char *name;
};
extern const MxConfig kMxConfigs[];
extern const int32_t kMxNumConfigs;
constexpr int32_t kMxDecode = 0, kMxDecode48 = 1;     // the decode kernel's rows
// Whether a configuration reads an A that is not loadable (below) where it lies; else it is copied first.
bool mx_direct_a(int32_t config, int64_t M, int64_t N, int64_t K);

// Whether the tile kernels take an operand as it lies (its first row at p, rows `stride` bytes
// apart) or have it copied first: they load 16 aligned bytes at a time straight into LDS, at
// 32-bit offsets within a tile.
constexpr int64_t kMxMostStride = int64_t(1) << 22;
inline bool mx_loadable(const void *p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 16 == 0 && stride <= kMxMostStride;
}

// Bytes of a row of A and of B's codes, on to the next multiple of 16.
inline int64_t mx_a_row(MxOp op, int64_t M, int64_t K) { return ((op == MX_DW ? M : K) * 2 + 15) / 16 * 16; }
inline int64_t mx_b_row(MxOp op, int64_t N, int64_t K) {
    return ((op == MX_FWD ? (K + 1) / 2 : op == MX_DX ? (N + 1) / 2 : N) + 15) / 16 * 16;
}

// The plan for a product, where `copied_a` and `copied_b` bytes of its operands are not loadable.
// config >= 0 and split > 0 say which one to evaluate instead.
// False where no configuration (the one named) is the operator's and takes the rows.
bool mx_select(MxOp op, int64_t M, int64_t N, int64_t K, int64_t copied_a, int64_t copied_b, int32_t config, int32_t split, MxPlan *out);

// Each queues its kernels on `stream` (a hipStream_t) and returns a LAUNCH_* value.
int launch_mx_pack(const MxMatrixArgs &a, int bits, void *stream);
int launch_mx_unpack(const MxMatrixArgs &a, int bits, void *stream);
int launch_mx_gemm(const MxArgs &a, MxOp op, const MxPlan &plan, void *stream);

}  // namespace gemm
