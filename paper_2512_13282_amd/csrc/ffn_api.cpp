// ffn_api.cpp -- the C ABI entry points of the gated feed-forward block (host side): argument
// checks before any HIP call, then the launch.
#include "../../include/ffn_mi355x.h"

#include <string.h>

#include "fused_api.h"

namespace {

using gemm::FusedArgs;
using gemm::FusedOp;
using gemm::Region;
using gemm::region;

constexpr FusedOp kOps[] = {gemm::FUSED_GATED, gemm::FUSED_GRAD, gemm::FUSED_DX, gemm::FUSED_DW, gemm::FUSED_DW};
constexpr int32_t kPairs[] = {1, 1, 1, 2, 1};
gemm::FusedForced g_forced[5];

bool known(int act) { return act >= FFN_SILU && act <= FFN_RELU; }

// The results against every operand and each other.
template <int I, int O>
bool sound(const Region (&in)[I], const Region (&out)[O]) {
    for (const Region &r : in)
        if (!r.valid()) return false;
    for (const Region &r : out)
        if (!r.valid()) return false;
    for (int o = 0; o < O; ++o) {
        for (const Region &r : in)
            if (out[o].overlaps(r)) return false;
        for (int p = 0; p < o; ++p)
            if (out[o].overlaps(out[p])) return false;
    }
    return true;
}

int launch(int op, FusedArgs &a, int64_t M, int64_t N, int64_t K, bool bf16_out, void *stream) {
    const bool at = kOps[op] == gemm::FUSED_DW, bt = kOps[op] == gemm::FUSED_GATED;
    const int64_t a_rows = at ? K : M, a_cols = at ? M : K, b_rows = bt ? N : K, b_cols = bt ? K : N;
    if (M > gemm::kFusedMostSize || N > gemm::kFusedMostSize || K > gemm::kFusedMostSize) return GEMM_ERR_UNSUPPORTED;
    const int64_t copied = gemm::fused_copied(a.g.A, a.g.lda, a_rows, a_cols, !at) + gemm::fused_copied(a.g.B, a.g.ldb, b_rows, b_cols, bt) +
                           (a.A2 != nullptr ? gemm::fused_copied(a.A2, a.lda2, a_rows, a_cols, !at) : 0) +
                           (a.B2 != nullptr ? gemm::fused_copied(a.B2, a.ldb2, b_rows, b_cols, bt) : 0);
    gemm::FusedPlan plan;
    const int planned = gemm::fused_plan_for(kOps[op], kPairs[op], M, N, K, copied, g_forced[op], &plan);
    if (planned != GEMM_OK) return planned;
    if (!gemm::fused_any_address(plan.config) && (!gemm::fused_copyable(a.g.A, a.g.lda, a_rows, a_cols, !at) || !gemm::fused_copyable(a.g.B, a.g.ldb, b_rows, b_cols, bt) ||
        (a.A2 != nullptr && !gemm::fused_copyable(a.A2, a.lda2, a_rows, a_cols, !at)) ||
        (a.B2 != nullptr && !gemm::fused_copyable(a.B2, a.ldb2, b_rows, b_cols, bt))))
        return GEMM_ERR_UNSUPPORTED;
    a.g.dtype = GEMM_DTYPE_BF16_F32;
    a.g.M = M;
    a.g.N = N;
    a.g.K = K;
    a.g.epilogue = bf16_out ? gemm::EPI_BF16 : gemm::EPI_NONE;
    a.pairs = kPairs[op];
    try {
        return gemm::fused_status(gemm::launch_fused(a, kOps[op], plan, stream));
    } catch (...) {      // the workspace table's own memory
        return GEMM_ERR_NO_MEMORY;
    }
}

int gated_dx(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *Wg, int64_t ldwg, const uint16_t *dU,
             int64_t lddu, const uint16_t *Wu, int64_t ldwu, void *dX, int64_t lddx, bool bf16_out, void *stream) {
    if (M < 0 || N < 0 || K < 0) return GEMM_ERR_INVALID_VALUE;
    const Region in[] = {region(dG, M, K, lddg, 2), region(Wg, K, N, ldwg, 2), region(dU, M, K, lddu, 2), region(Wu, K, N, ldwu, 2)};
    const Region out[] = {region(dX, M, N, lddx, bf16_out ? 2 : 4)};
    if (!sound(in, out)) return GEMM_ERR_INVALID_VALUE;
    if (M == 0 || N == 0) return GEMM_OK;
    FusedArgs a{};
    a.g.A = dG; a.g.lda = lddg;
    a.g.B = Wg; a.g.ldb = ldwg;
    a.A2 = dU; a.lda2 = lddu;
    a.B2 = Wu; a.ldb2 = ldwu;
    a.g.C = dX; a.g.ldc = lddx;
    return launch(FFN_OP_DX, a, M, N, K, bf16_out, stream);
}

int dw(int op, int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *dU, int64_t lddu, const uint16_t *X,
       int64_t ldx, void *dWg, int64_t lddwg, void *dWu, int64_t lddwu, bool bf16_out, void *stream) {
    if (M < 0 || N < 0 || K < 0) return GEMM_ERR_INVALID_VALUE;
    const int64_t second = op == FFN_OP_GATED_DW ? 1 : 0, size = bf16_out ? 2 : 4;
    const Region in[] = {region(dG, K, M, lddg, 2), region(dU, second * K, M, lddu, 2), region(X, K, N, ldx, 2)};
    const Region out[] = {region(dWg, M, N, lddwg, size), region(dWu, second * M, N, lddwu, size)};
    if (!sound(in, out)) return GEMM_ERR_INVALID_VALUE;
    if (M == 0 || N == 0) return GEMM_OK;
    FusedArgs a{};
    a.g.A = dG; a.g.lda = lddg;
    a.A2 = dU; a.lda2 = lddu;
    a.g.B = X; a.g.ldb = ldx;
    a.g.C = dWg; a.g.ldc = lddwg;
    a.C2 = dWu; a.ldc2 = lddwu;
    return launch(op, a, M, N, K, bf16_out, stream);
}

}  // namespace

extern "C" {

int ffn_gated_bf16_bt(int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx, const uint16_t *Wg, int64_t ldwg, const uint16_t *Wu,
                      int64_t ldwu, int act, uint16_t *H, int64_t ldh, uint16_t *G, int64_t ldg, uint16_t *U, int64_t ldu, void *stream) {
    if (M < 0 || N < 0 || K < 0 || !known(act)) return GEMM_ERR_INVALID_VALUE;
    const bool some = M > 0 && N > 0;
    if (some && (G == nullptr) != (U == nullptr)) return GEMM_ERR_INVALID_VALUE;
    const int64_t kept = G != nullptr ? M : 0;
    const Region in[] = {region(X, M, K, ldx, 2), region(Wg, N, K, ldwg, 2), region(Wu, N, K, ldwu, 2)};
    const Region out[] = {region(H, M, N, ldh, 2), region(G, kept, N, ldg, 2), region(U, kept, N, ldu, 2)};
    if (!sound(in, out)) return GEMM_ERR_INVALID_VALUE;
    if (!some) return GEMM_OK;
    FusedArgs a{};
    a.g.A = X; a.g.lda = ldx;
    a.g.B = Wg; a.g.ldb = ldwg;
    a.B2 = Wu; a.ldb2 = ldwu;
    a.act = act;
    a.g.C = H; a.g.ldc = ldh;
    a.C2 = G; a.ldc2 = ldg;
    a.C3 = U; a.ldc3 = ldu;
    return launch(FFN_OP_GATED, a, M, N, K, true, stream);
}

int ffn_gated_grad_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *Wd, int64_t ldwd, const uint16_t *G,
                        int64_t ldg, const uint16_t *U, int64_t ldu, int act, uint16_t *dG, int64_t lddg, uint16_t *dU, int64_t lddu,
                        uint16_t *H, int64_t ldh, void *stream) {
    if (M < 0 || N < 0 || K < 0 || !known(act)) return GEMM_ERR_INVALID_VALUE;
    const Region in[] = {region(dY, M, K, lddy, 2), region(Wd, K, N, ldwd, 2), region(G, M, N, ldg, 2), region(U, M, N, ldu, 2)};
    const Region out[] = {region(dG, M, N, lddg, 2), region(dU, M, N, lddu, 2), region(H, H != nullptr ? M : 0, N, ldh, 2)};
    if (!sound(in, out)) return GEMM_ERR_INVALID_VALUE;
    if (M == 0 || N == 0) return GEMM_OK;
    FusedArgs a{};
    a.g.A = dY; a.g.lda = lddy;
    a.g.B = Wd; a.g.ldb = ldwd;
    a.G = G; a.ldg = ldg;
    a.U = U; a.ldu = ldu;
    a.act = act;
    a.g.C = dG; a.g.ldc = lddg;
    a.C2 = dU; a.ldc2 = lddu;
    a.C3 = H; a.ldc3 = ldh;
    return launch(FFN_OP_GRAD, a, M, N, K, true, stream);
}

int ffn_gated_bwd_bf16(int64_t M, int64_t N, const uint16_t *dH, int64_t lddh, const uint16_t *G, int64_t ldg, const uint16_t *U, int64_t ldu,
                       int act, uint16_t *dG, int64_t lddg, uint16_t *dU, int64_t lddu, void *stream) {
    if (M < 0 || N < 0 || !known(act)) return GEMM_ERR_INVALID_VALUE;
    const Region in[] = {region(dH, M, N, lddh, 2), region(G, M, N, ldg, 2), region(U, M, N, ldu, 2)};
    const Region out[] = {region(dG, M, N, lddg, 2), region(dU, M, N, lddu, 2)};
    if (!sound(in, out)) return GEMM_ERR_INVALID_VALUE;
    if (M == 0 || N == 0) return GEMM_OK;
    return gemm::fused_status(gemm::launch_gated_bwd({M, N, dH, G, U, dG, dU, lddh, ldg, ldu, lddg, lddu, act}, stream));
}

int ffn_gated_dx_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *Wg, int64_t ldwg, const uint16_t *dU,
                     int64_t lddu, const uint16_t *Wu, int64_t ldwu, float *dX, int64_t lddx, void *stream) {
    return gated_dx(M, N, K, dG, lddg, Wg, ldwg, dU, lddu, Wu, ldwu, dX, lddx, false, stream);
}

int ffn_gated_dx_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *Wg, int64_t ldwg, const uint16_t *dU,
                      int64_t lddu, const uint16_t *Wu, int64_t ldwu, uint16_t *dX, int64_t lddx, void *stream) {
    return gated_dx(M, N, K, dG, lddg, Wg, ldwg, dU, lddu, Wu, ldwu, dX, lddx, true, stream);
}

int ffn_gated_dw_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *dU, int64_t lddu, const uint16_t *X,
                     int64_t ldx, float *dWg, int64_t lddwg, float *dWu, int64_t lddwu, void *stream) {
    return dw(FFN_OP_GATED_DW, M, N, K, dG, lddg, dU, lddu, X, ldx, dWg, lddwg, dWu, lddwu, false, stream);
}

int ffn_gated_dw_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dG, int64_t lddg, const uint16_t *dU, int64_t lddu, const uint16_t *X,
                      int64_t ldx, uint16_t *dWg, int64_t lddwg, uint16_t *dWu, int64_t lddwu, void *stream) {
    return dw(FFN_OP_GATED_DW, M, N, K, dG, lddg, dU, lddu, X, ldx, dWg, lddwg, dWu, lddwu, true, stream);
}

int ffn_dw_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *X, int64_t ldx, float *dW, int64_t lddw,
               void *stream) {
    return dw(FFN_OP_DW, M, N, K, dY, lddy, nullptr, 0, X, ldx, dW, lddw, nullptr, 0, false, stream);
}

int ffn_dw_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *X, int64_t ldx, uint16_t *dW, int64_t lddw,
                void *stream) {
    return dw(FFN_OP_DW, M, N, K, dY, lddy, nullptr, 0, X, ldx, dW, lddw, nullptr, 0, true, stream);
}

int ffn_plan(int op, int64_t M, int64_t N, int64_t K, ffn_plan_info *out) {
    if (out == nullptr || op < FFN_OP_GATED || op > FFN_OP_DW || M < 0 || N < 0 || K < 0) return GEMM_ERR_INVALID_VALUE;
    memset(out, 0, sizeof(*out));
    out->config = -1;
    if (M == 0 || N == 0) return GEMM_OK;
    gemm::FusedPlan plan;
    const int rc = gemm::fused_plan_for(kOps[op], kPairs[op], M, N, K, 0, g_forced[op], &plan);
    if (rc != GEMM_OK) return rc;
    const gemm::FusedConfig &c = gemm::kFusedConfigs[plan.config];
    out->config = plan.config;
    out->bm = c.bm;
    out->bn = op == FFN_OP_GATED ? c.bn / 2 : c.bn;
    out->split_k = plan.split_k;
    out->k_chunk = plan.k_chunk;
    strncpy(out->name, c.name, sizeof(out->name) - 1);
    return GEMM_OK;
}

int ffn_force_plan(int op, int config, int split_k) {
    if (op < FFN_OP_GATED || op > FFN_OP_DW || config < -1 || split_k < 0 || (config >= 0 && !gemm::fused_has(kOps[op], config)))
        return GEMM_ERR_INVALID_VALUE;
    g_forced[op].config = config;
    g_forced[op].split = split_k;
    return GEMM_OK;
}

}  // extern "C"
