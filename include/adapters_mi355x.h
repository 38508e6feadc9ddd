/*
 * adapters_mi355x.h -- C ABI of the MI355X (gfx950) projection that many requests share, each with a
 * low-rank adapter of its own, and its gradients.
 *
 * A weight W (out x in), n adapters of rank r, A_i (r x in) and B_i (out x r), and a scale s_i each.  Token t has
 * adapter index[t] where that lies in [0, n), and none where it does not (-1, say); tokens may be in any order:
 *
 *   h_t = s_i x_t A_i^T,     y_t = x_t W^T + h_t B_i^T
 *   dh_t = s_i dy_t B_i,     dx_t = dy_t W + dh_t A_i
 *   dA_i = sum_t dh_t^T x_t,  dB_i = sum_t dy_t^T h_t        over the tokens of adapter i
 *
 * x, dy, W, A and B are bf16, the scales fp32, h and dh fp32 (M x r, rows r apart; zeros for a token without an
 * adapter), the index 32-bit integers, all in DEVICE memory.  Products are exact and accumulated in fp32;
 * between the two products of an adapter nothing is rounded to fewer than 16 bits where the result is bf16, and to
 * fewer than 24 where it is fp32.  What a request's adapter holds, infinities and NaN included, reaches that
 * request's rows alone, and is there what the formula makes of it.  Results do not depend on the order in which workgroups run.
 *
 * Ownership, workspaces, streams, capture, realigned operands and error codes are those of ffn_mi355x.h.  A captured
 * call reads the index, the scales and the adapters anew at each replay.  GEMM_ERR_INVALID_VALUE is returned for a
 * NULL set, a negative n or r, and an adapter's matrix that overlaps the next one, too, and GEMM_ERR_UNSUPPORTED for a
 * rank above 1024, too; by adapters_linear_* for more than 2^26 tokens or 2^31 - 1 adapters, by adapters_dw_* for more than 65535
 * adapters or N + K above 2^29.  A, B and the adapters' gradients may lie at any address and stride.
 */
#ifndef ADAPTERS_MI355X_H
#define ADAPTERS_MI355X_H

#include <stdint.h>

#include "gemm_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct adapters_set {
    int64_t n, r;
    const uint16_t *A;        /* n matrices r x in, rows lda and adapters sa elements apart   */
    int64_t lda, sa;
    const uint16_t *B;        /* n matrices out x r, rows ldb and adapters sb elements apart  */
    int64_t ldb, sb;
    const float *scale;       /* n of them, or NULL: 1                                        */
} adapters_set;

/* Y (M x N) = x W^T + the adapters' part: X M x K (K inputs), W N x K (N outputs).  H: h (M x r), or NULL. */
int adapters_linear_f32_bt(int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx, const uint16_t *W, int64_t ldw,
                           const adapters_set *set, const int32_t *index, float *Y, int64_t ldy, float *H, void *stream);
int adapters_linear_bf16_bt(int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx, const uint16_t *W, int64_t ldw,
                            const adapters_set *set, const int32_t *index, uint16_t *Y, int64_t ldy, float *H, void *stream);

/* dX (M x N) = dy W + the adapters' part: dY M x K (K outputs), W K x N (N inputs).  dH: dh (M x r), or NULL. */
int adapters_linear_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *W, int64_t ldw,
                        const adapters_set *set, const int32_t *index, float *dX, int64_t lddx, float *dH, void *stream);
int adapters_linear_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *W, int64_t ldw,
                         const adapters_set *set, const int32_t *index, uint16_t *dX, int64_t lddx, float *dH, void *stream);

/* dA (n matrices r x K) and dB (n matrices N x r) of M tokens, X M x K, dY M x N; zeros for an adapter without tokens. */
int adapters_dw_f32(int64_t M, int64_t N, int64_t K, int64_t n, int64_t r, const uint16_t *X, int64_t ldx,
                    const uint16_t *dY, int64_t lddy, const float *H, const float *dH, const int32_t *index,
                    float *dA, int64_t ldda, int64_t sda, float *dB, int64_t lddb, int64_t sdb, void *stream);
int adapters_dw_bf16(int64_t M, int64_t N, int64_t K, int64_t n, int64_t r, const uint16_t *X, int64_t ldx,
                     const uint16_t *dY, int64_t lddy, const float *H, const float *dH, const int32_t *index,
                     uint16_t *dA, int64_t ldda, int64_t sda, uint16_t *dB, int64_t lddb, int64_t sdb, void *stream);

/* Test and benchmark hook, as ffn_force_plan: the products with W. */
enum { ADAPTERS_OP_FORWARD = 0, ADAPTERS_OP_INPUT_GRADIENT = 1 };
int adapters_force_plan(int op, int config, int split_k);

#ifdef __cplusplus
}
#endif

#endif /* ADAPTERS_MI355X_H */
