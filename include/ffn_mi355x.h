/*
 * ffn_mi355x.h -- C ABI of the MI355X (gfx950) gated feed-forward block and its gradients.
 *
 * A block with gate and up projections Wg, Wu and a down projection Wd computes
 *
 *   G = X Wg^T,   U = X Wu^T,   H = act(G) * U,   Y = H Wd^T
 *
 * (Y by gemm_bf16_*_bt).  Operands are bf16, row-major, row strides in ELEMENTS; products are exact
 * and accumulated in fp32, and each result is rounded once, to the nearest bf16, ties to even
 * (the f32 forms are not rounded).  Results overwrite; row padding is never touched.
 *
 * Ownership, workspaces, streams, capture and error codes are those of gemm_mi355x.h: operands are caller-owned
 * DEVICE pointers on the current device, every call is asynchronous on `stream` and may be captured
 * (its replays ordered with that stream's other calls), argument checks run on the host before any HIP call, no
 * entry point throws or aborts, and workspaces (partial sums of K slices, realigned copies) are the
 * ones that gemm_release_workspace frees.  Reads are made in pieces of up to 16 bytes: an operand
 * whose rows lie on 16-byte addresses may have the bytes up to its row's next multiple of 16 read,
 * any other the rest of the aligned four bytes that hold a row's first and last element, without being used.
 * GEMM_ERR_INVALID_VALUE is returned for a negative size, a stride that is too small, a NULL pointer
 * whose operand is non-empty, a pointer that is not aligned to its element size, an unknown
 * activation, and a result that overlaps an operand or another result; GEMM_ERR_UNSUPPORTED for a size
 * of 2^31 - 4096 or more, for more output tiles than a launch holds, and for rows that have to be
 * copied and are longer than 4 MiB.
 * Operands are read where they lie if their address and row stride are multiples of 16 bytes, the stride at most 4 MiB,
 * and, of those whose rows lie along the sum, if the rows are whole multiples of 16 bytes; other operands are
 * copied to such rows first, in the stream's workspace, which keeps the size of the
 * largest such copies until gemm_release_workspace.
 * A size of 0 of the results is a successful no-op; an empty sum is 0.
 */
#ifndef FFN_MI355X_H
#define FFN_MI355X_H

#include <stdint.h>

#include "gemm_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

/* act(g): g / (1 + e^-g); g P(g) with P the standard normal distribution; g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2;
 * max(g, 0).  A NaN stays one.  The derivative of the last at 0 is 0.  Values of act and act' below 2^-100 may be taken
 * for 0. */
enum { FFN_SILU = 0, FFN_GELU = 1, FFN_GELU_TANH = 2, FFN_RELU = 3 };

/* H (M x N) = act(X Wg^T) * (X Wu^T), X M x K, Wg and Wu N x K.  G and U (M x N each): where they are not NULL (both or
 * neither), X Wg^T and X Wu^T rounded to bf16, for the backward pass; H is formed from the sums themselves. */
int ffn_gated_bf16_bt(int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx,
                      const uint16_t *Wg, int64_t ldwg, const uint16_t *Wu, int64_t ldwu, int act,
                      uint16_t *H, int64_t ldh, uint16_t *G, int64_t ldg, uint16_t *U, int64_t ldu, void *stream);

/* The gradients of G and U (M x N) from dY (M x K) and Wd (K x N), with dH = dY Wd kept in fp32:
 * dG = dH * U * act'(G), dU = dH * act(G); and, where H is not NULL, H = act(G) * U from the kept G and U, which the
 * gradient of Wd takes. */
int ffn_gated_grad_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *Wd, int64_t ldwd,
                        const uint16_t *G, int64_t ldg, const uint16_t *U, int64_t ldu, int act,
                        uint16_t *dG, int64_t lddg, uint16_t *dU, int64_t lddu, uint16_t *H, int64_t ldh, void *stream);

/* The same from the gradient dH of H itself (M x N, bf16), where something else than a projection follows:
 * dG = dH * U * act'(G), dU = dH * act(G), for any dH. */
int ffn_gated_bwd_bf16(int64_t M, int64_t N, const uint16_t *dH, int64_t lddh, const uint16_t *G, int64_t ldg,
                       const uint16_t *U, int64_t ldu, int act, uint16_t *dG, int64_t lddg, uint16_t *dU, int64_t lddu, void *stream);

/* dX (M x N) = dG Wg + dU Wu, dG and dU M x K, Wg and Wu K x N: both products in one sum. */
int ffn_gated_dx_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *Wg, int64_t ldwg,
                     const uint16_t *dU, int64_t lddu, const uint16_t *Wu, int64_t ldwu, float *dX, int64_t lddx, void *stream);
int ffn_gated_dx_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *Wg, int64_t ldwg,
                      const uint16_t *dU, int64_t lddu, const uint16_t *Wu, int64_t ldwu, uint16_t *dX, int64_t lddx, void *stream);

/* dWg = dG^T X and dWu = dU^T X (M x N each), dG and dU K x M, X K x N: K tokens, M outputs and N inputs of the weights. */
int ffn_gated_dw_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *dU, int64_t lddu,
                     const uint16_t *X, int64_t ldx, float *dWg, int64_t lddwg, float *dWu, int64_t lddwu, void *stream);
int ffn_gated_dw_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *dU, int64_t lddu,
                      const uint16_t *X, int64_t ldx, uint16_t *dWg, int64_t lddwg, uint16_t *dWu, int64_t lddwu, void *stream);

/* dW (M x N) = dY^T X, dY K x M, X K x N: the weight gradient of one projection. */
int ffn_dw_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *X, int64_t ldx,
               float *dW, int64_t lddw, void *stream);
int ffn_dw_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *X, int64_t ldx,
                uint16_t *dW, int64_t lddw, void *stream);

/* Pure host: the plan that a call of these sizes uses, its operands on 16-byte rows: the kernel's configuration (-1: nothing
 * to do), its output tile (GATED: of H), the number of K slices of the tiles that fill no whole round of the compute units,
 * and the K of each (the gradient of X: of both products, one after the other, each on whole 64 k).
 * GEMM_ERR_INVALID_VALUE: an unknown op, a negative size, a NULL out. */
typedef struct ffn_plan_info {
    int32_t config;
    int32_t bm, bn;
    int32_t split_k;
    int64_t k_chunk;
    char    name[48];
} ffn_plan_info;

enum { FFN_OP_GATED = 0, FFN_OP_GRAD = 1, FFN_OP_DX = 2, FFN_OP_GATED_DW = 3, FFN_OP_DW = 4 };

int ffn_plan(int op, int64_t M, int64_t N, int64_t K, ffn_plan_info *out);

/* Test and benchmark hook: the configuration (-1: the library's choice) and the number of K slices (0: its choice) of
 * every later call of `op`.  A call that the configuration cannot run returns GEMM_ERR_UNSUPPORTED. */
int ffn_force_plan(int op, int config, int split_k);

#ifdef __cplusplus
}
#endif

#endif /* FFN_MI355X_H */
