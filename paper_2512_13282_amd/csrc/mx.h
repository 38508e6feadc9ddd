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

// Each queues its kernels on `stream` (a hipStream_t) and returns a LAUNCH_* value.
int launch_mx_pack(const MxMatrixArgs &a, int bits, void *stream);
int launch_mx_unpack(const MxMatrixArgs &a, int bits, void *stream);
int launch_mx_gemm(const MxArgs &a, MxOp op, void *stream);

}  // namespace gemm
