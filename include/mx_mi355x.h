/*
 * mx_mi355x.h -- C ABI of the MI355X (gfx950) products over block-scaled operands:
 * linear layers whose weight is held in 4 bits, activation checkpoints in 8 bits.
 *
 * Formats (the OCP Microscaling formats MXFP4 and MXINT8; the latter's specification
 * takes a code for a multiple of 2^-6, here it is a whole number, so the same matrix has
 * scale bytes 6 smaller here).  A packed matrix of `rows` x `cols` elements has two parts:
 *
 *   scales  one byte e for every block of 32 consecutive elements of a row (the
 *           row's last block may be shorter), the power of two 2^(e - 127); e = 255
 *           makes every element of the block NaN.  Row stride lds, in bytes, at
 *           least ceil(cols / 32).
 *   codes   4 bits: an element is the E2M1 number of sign, two exponent bits and one
 *           mantissa bit (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a
 *           byte, the first in the low half; row stride ldq, in BYTES, at least
 *           ceil(cols / 2).
 *           8 bits: an element is a signed byte, written in [-127, 127]; row stride
 *           ldq, in bytes, at least cols.
 *
 * An element stands for (its code's value) * (its block's scale).  Every such value is a
 * bf16 number exactly, but for those past bf16's range, which count as infinities of
 * their sign: code values of 2^(255 - e) and more (4 bits: under bytes 253 and 254; 8
 * bits: from 248 on).  Packing makes none of them.
 * The products below work on these values themselves: products are exact and are
 * accumulated in fp32, as gemm_bf16_f32's.
 *
 * Ownership, workspaces, streams, capture and error codes are those of
 * gemm_mi355x.h: operands are caller-owned DEVICE pointers on the current device,
 * every call is asynchronous on `stream` and may be captured, argument checks run on
 * the host before any HIP call, no entry point throws or aborts, and workspaces
 * (split-K partials, realigned copies) are the ones that gemm_release_workspace
 * frees.  Reads are made in aligned pieces of up to 16 bytes: a row's last piece may
 * read, without using, the bytes up to the next multiple of 16.
 * GEMM_ERR_INVALID_VALUE is returned for a negative size, a stride that is too small,
 * a NULL pointer whose operand is non-empty, a bf16 or fp32 pointer that is not
 * aligned to its element size, and an output that overlaps an input or another output;
 * GEMM_ERR_UNSUPPORTED for a product with a size of 2^31 - 4096 or more, with more output
 * tiles than a launch holds (2^23 workgroups of 512 threads), or with rows of A,
 * At or the codes longer than 4 MiB (up to 48 rows of A over W^T take K up to 1.1 * 10^8 / M).
 * Operands whose rows do not lie on 16-byte addresses are copied to rows that do, in the
 * stream's workspace, ahead of a product (but for a few rows of A over W^T, and A and At
 * where the results have few rows).  The workspace keeps the size of the largest such
 * copies, and while it grows the buffers that it replaces, until gemm_release_workspace:
 * codes with ldq and their address multiples of 16 cost no memory.
 */
#ifndef MX_MI355X_H
#define MX_MI355X_H

#include <stdint.h>

#include "gemm_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Packs the bf16 matrix X (rows x cols, row stride ldx in elements).  The scale of a
 * block whose largest magnitude lies in [2^x, 2^(x+1)) is 2^(x - 2) (4 bits) or
 * 2^(x - 6) (8 bits), at least 2^-127; an element is its value over the scale rounded
 * to the nearest code, ties to even, and saturated (at 6 resp. 127).  A block of
 * zeros takes e = 0; one that holds an infinity or a NaN takes e = 255 and codes 0.
 * The unused half of a last byte is 0.  Bytes of a row past its last code and scale
 * are not touched. */
int mx_pack4(int64_t rows, int64_t cols, const uint16_t *X, int64_t ldx,
             uint8_t *codes, int64_t ldq, uint8_t *scales, int64_t lds, void *stream);
int mx_pack8(int64_t rows, int64_t cols, const uint16_t *X, int64_t ldx,
             int8_t *codes, int64_t ldq, uint8_t *scales, int64_t lds, void *stream);

/* The bf16 matrix that packed codes stand for, exactly. */
int mx_unpack4(int64_t rows, int64_t cols, const uint8_t *codes, int64_t ldq,
               const uint8_t *scales, int64_t lds, uint16_t *X, int64_t ldx, void *stream);
int mx_unpack8(int64_t rows, int64_t cols, const int8_t *codes, int64_t ldq,
               const uint8_t *scales, int64_t lds, uint16_t *X, int64_t ldx, void *stream);

/* C (M x N, row stride ldc) = A (M x K bf16, row stride lda) . W^T, W a 4-bit matrix of
 * N x K: a linear layer over its weight, from one row (a token) up.  fp32 results, or
 * rounded once to the nearest bf16, ties to even. */
int mx_gemm_bf16_mx4_f32_bt(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda,
                            const uint8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
                            float *C, int64_t ldc, void *stream);
int mx_gemm_bf16_mx4_bf16_bt(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda,
                             const uint8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
                             uint16_t *C, int64_t ldc, void *stream);

/* C (M x N) = A (M x K bf16) . W, W a 4-bit matrix of K x N (blocks along N): the input
 * gradient dX = dY . W of the same layer, over the same packed weight. */
int mx_gemm_bf16_mx4_f32(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda,
                         const uint8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
                         float *C, int64_t ldc, void *stream);
int mx_gemm_bf16_mx4_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda,
                          const uint8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
                          uint16_t *C, int64_t ldc, void *stream);

/* C (M x N) = At^T . X, At a bf16 matrix of K x M (row stride ldat) and X an 8-bit matrix
 * of K x N: the weight gradient dW = dY^T . X of a layer of M outputs and N inputs over
 * K tokens, from the layer's packed input. */
int mx_gemm_bf16_mx8_f32_at(int64_t M, int64_t N, int64_t K, const uint16_t *At, int64_t ldat,
                            const int8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
                            float *C, int64_t ldc, void *stream);
int mx_gemm_bf16_mx8_bf16_at(int64_t M, int64_t N, int64_t K, const uint16_t *At, int64_t ldat,
                             const int8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
                             uint16_t *C, int64_t ldc, void *stream);

/* Pure host: the plan that a product of these sizes, its operands on aligned rows, would use: the kernel's
 * configuration (-1: nothing to do), its output tile, the number of K slices and the K
 * of each.  GEMM_ERR_INVALID_VALUE: an unknown op, a negative size, a NULL out. */
typedef struct mx_plan_info {
    int32_t config;
    int32_t bm, bn;
    int32_t split_k;
    int64_t k_chunk;
    char    name[48];
} mx_plan_info;

enum { MX_OP_FORWARD = 0, MX_OP_INPUT_GRADIENT = 1, MX_OP_WEIGHT_GRADIENT = 2 };

int mx_plan(int op, int64_t M, int64_t N, int64_t K, mx_plan_info *out);

/* Test and benchmark hook: the configuration (-1: the library's choice) and the number of
 * K slices (0: its choice) of every later product of `op`.  A product that the
 * configuration cannot run returns GEMM_ERR_UNSUPPORTED. */
int mx_force_plan(int op, int config, int split_k);

#ifdef __cplusplus
}
#endif

#endif /* MX_MI355X_H */
