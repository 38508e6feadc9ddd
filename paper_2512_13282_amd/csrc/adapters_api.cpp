// adapters_api.cpp -- the C ABI entry points of the projection with adapters (host side): argument
// checks before any HIP call, then the launch.
#include "../../include/adapters_mi355x.h"

#include "adapters.h"
#include "fused_api.h"

namespace {

using gemm::Region;
using gemm::region;

gemm::FusedForced g_forced[2];

// n matrices of rows x cols, `stride` elements from one to the next: one region, and whether they lie apart.
struct Stack {
    Region all;
    bool apart;
    bool valid() const { return apart && all.valid(); }
};
Stack stack(const void *p, int64_t n, int64_t rows, int64_t cols, int64_t ld, int64_t stride, int64_t size) {
    const Region one = region(p, n > 0 ? rows : 0, cols, ld, size);
    if (one.empty()) return {one, true};
    if (!one.valid() || n > gemm::kMaxSize || stride > gemm::kMaxSize) return {one, false};
    const int64_t span = int64_t(one.span());
    if (n > 1 && (stride < 0 || stride * size < span || stride * size > gemm::kMaxSize / n)) return {one, false};
    return {Region{one.p, n, span, n > 1 ? stride * size : span, size}, true};
}

int product(int op, int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx, const uint16_t *W, int64_t ldw, const adapters_set *set,
            const int32_t *index, void *Y, int64_t ldy, float *H, bool bf16_out, void *stream) {
    const bool forward = op == ADAPTERS_OP_FORWARD;
    if (M < 0 || N < 0 || K < 0 || set == nullptr || set->n < 0 || set->r < 0) return GEMM_ERR_INVALID_VALUE;
    const int64_t n = set->n, r = set->r;
    const bool some = n > 0 && r > 0;
    const Region rx = region(X, M, K, ldx, 2), rw = forward ? region(W, N, K, ldw, 2) : region(W, K, N, ldw, 2);
    const Region ry = region(Y, M, N, ldy, bf16_out ? 2 : 4), rh = region(H, H != nullptr && r > 0 ? M : 0, r, r, 4);
    const Region ri = region(index, some ? 1 : 0, M, M, 4), rs = region(set->scale, some && set->scale != nullptr ? 1 : 0, n, n, 4);
    const Stack A = stack(set->A, n, r, forward ? K : N, set->lda, set->sa, 2), B = stack(set->B, n, forward ? N : K, r, set->ldb, set->sb, 2);
    if (!rx.valid() || !rw.valid() || !ry.valid() || !rh.valid() || !ri.valid() || !rs.valid() || !A.valid() || !B.valid())
        return GEMM_ERR_INVALID_VALUE;
    const Region in[] = {rx, rw, ri, rs, A.all, B.all};
    for (const Region &i : in)
        if (ry.overlaps(i) || rh.overlaps(i)) return GEMM_ERR_INVALID_VALUE;
    if (ry.overlaps(rh)) return GEMM_ERR_INVALID_VALUE;
    if (n > INT32_MAX || r > gemm::kAdaptersMostRank || M > (int64_t(1) << 26)) return GEMM_ERR_UNSUPPORTED;
    if (M == 0 || (N == 0 && rh.empty())) return GEMM_OK;
    gemm::FusedArgs a{};
    gemm::FusedPlan plan{};
    const gemm::FusedOp fused = forward ? gemm::FUSED_ADAPT : gemm::FUSED_ADAPT_DX;
    if (K > gemm::kFusedMostSize) return GEMM_ERR_UNSUPPORTED;
    if (N > gemm::kFusedMostSize) return GEMM_ERR_UNSUPPORTED;
    if (N > 0) {
        const int64_t copied = gemm::fused_copied(X, ldx, M, K, true) + gemm::fused_copied(W, ldw, forward ? N : K, forward ? K : N, forward);
        const int planned = gemm::fused_plan_for(fused, 1, M, N, K, copied, g_forced[op], &plan);
        if (planned != GEMM_OK) return planned;
        if (!gemm::fused_any_address(plan.config) &&
            (!gemm::fused_copyable(X, ldx, M, K, true) || !gemm::fused_copyable(W, ldw, forward ? N : K, forward ? K : N, forward)))
            return GEMM_ERR_UNSUPPORTED;
    }
    a.g.dtype = GEMM_DTYPE_BF16_F32;
    a.g.A = X; a.g.lda = ldx;
    a.g.B = W; a.g.ldb = ldw;
    a.g.C = Y; a.g.ldc = ldy;
    a.g.M = M; a.g.N = N; a.g.K = K;
    a.g.epilogue = bf16_out ? gemm::EPI_BF16 : gemm::EPI_NONE;
    a.pairs = 1;
    a.n = int32_t(n);
    a.r = int32_t(r);
    a.index = index;
    a.Q = forward ? set->B : set->A;
    a.ldq = forward ? set->ldb : set->lda;
    a.sq = forward ? set->sb : set->sa;
    gemm::ShrinkArgs s{};
    s.P = X; s.ldp = ldx;
    s.M = M; s.L = K;
    s.Q = forward ? set->A : set->B;
    s.ldq = forward ? set->lda : set->ldb;
    s.sq = forward ? set->sa : set->sb;
    s.scale = set->scale;
    s.index = index;
    s.n = a.n;
    s.r = a.r;
    s.qt = forward;
    s.h = H;
    try {
        return gemm::fused_status(gemm::launch_adapters(a, fused, plan, s, stream));
    } catch (...) {      // the workspace table's own memory
        return GEMM_ERR_NO_MEMORY;
    }
}

int gradients(int64_t M, int64_t N, int64_t K, int64_t n, int64_t r, const uint16_t *X, int64_t ldx, const uint16_t *dY, int64_t lddy,
              const float *H, const float *dH, const int32_t *index, void *dA, int64_t ldda, int64_t sda, void *dB, int64_t lddb, int64_t sdb,
              bool bf16_out, void *stream) {
    if (M < 0 || N < 0 || K < 0 || n < 0 || r < 0) return GEMM_ERR_INVALID_VALUE;
    const int64_t rows = n > 0 && r > 0 ? M : 0, size = bf16_out ? 2 : 4;
    const Region in[] = {region(X, rows, K, ldx, 2), region(dY, rows, N, lddy, 2), region(H, N > 0 ? rows : 0, r, r, 4),
                         region(dH, K > 0 ? rows : 0, r, r, 4), region(index, K > 0 || N > 0 ? (rows > 0 ? 1 : 0) : 0, M, M, 4)};
    const Stack a = stack(dA, n, r, K, ldda, sda, size), b = stack(dB, n, N, r, lddb, sdb, size);
    if (!a.valid() || !b.valid() || a.all.overlaps(b.all)) return GEMM_ERR_INVALID_VALUE;
    for (const Region &i : in)
        if (!i.valid() || a.all.overlaps(i) || b.all.overlaps(i)) return GEMM_ERR_INVALID_VALUE;
    if (n > 65535 || r > gemm::kAdaptersMostRank || M > gemm::kFusedMostSize || N + K > (int64_t(1) << 29)) return GEMM_ERR_UNSUPPORTED;
    if (n == 0 || r == 0 || (N == 0 && K == 0)) return GEMM_OK;
    gemm::AdapterDwArgs g{};
    g.M = M;
    g.n = int32_t(n);
    g.r = int32_t(r);
    g.index = index;
    g.side[0] = {X, ldx, K, dH, dA, ldda, sda, int32_t((K + 63) / 64)};
    g.side[1] = {dY, lddy, N, H, dB, lddb, sdb, int32_t((N + 63) / 64)};
    g.bf16_out = bf16_out ? 1 : 0;
    return gemm::fused_status(gemm::launch_adapters_dw(g, stream));
}

}  // namespace

extern "C" {

int adapters_linear_f32_bt(int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx, const uint16_t *W, int64_t ldw,
                           const adapters_set *set, const int32_t *index, float *Y, int64_t ldy, float *H, void *stream) {
    return product(ADAPTERS_OP_FORWARD, M, N, K, X, ldx, W, ldw, set, index, Y, ldy, H, false, stream);
}

int adapters_linear_bf16_bt(int64_t M, int64_t N, int64_t K, const uint16_t *X, int64_t ldx, const uint16_t *W, int64_t ldw,
                            const adapters_set *set, const int32_t *index, uint16_t *Y, int64_t ldy, float *H, void *stream) {
    return product(ADAPTERS_OP_FORWARD, M, N, K, X, ldx, W, ldw, set, index, Y, ldy, H, true, stream);
}

int adapters_linear_f32(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *W, int64_t ldw,
                        const adapters_set *set, const int32_t *index, float *dX, int64_t lddx, float *dH, void *stream) {
    return product(ADAPTERS_OP_INPUT_GRADIENT, M, N, K, dY, lddy, W, ldw, set, index, dX, lddx, dH, false, stream);
}

int adapters_linear_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *dY, int64_t lddy, const uint16_t *W, int64_t ldw,
                         const adapters_set *set, const int32_t *index, uint16_t *dX, int64_t lddx, float *dH, void *stream) {
    return product(ADAPTERS_OP_INPUT_GRADIENT, M, N, K, dY, lddy, W, ldw, set, index, dX, lddx, dH, true, stream);
}

int adapters_dw_f32(int64_t M, int64_t N, int64_t K, int64_t n, int64_t r, const uint16_t *X, int64_t ldx, const uint16_t *dY, int64_t lddy,
                    const float *H, const float *dH, const int32_t *index, float *dA, int64_t ldda, int64_t sda, float *dB, int64_t lddb,
                    int64_t sdb, void *stream) {
    return gradients(M, N, K, n, r, X, ldx, dY, lddy, H, dH, index, dA, ldda, sda, dB, lddb, sdb, false, stream);
}

int adapters_dw_bf16(int64_t M, int64_t N, int64_t K, int64_t n, int64_t r, const uint16_t *X, int64_t ldx, const uint16_t *dY, int64_t lddy,
                     const float *H, const float *dH, const int32_t *index, uint16_t *dA, int64_t ldda, int64_t sda, uint16_t *dB, int64_t lddb,
                     int64_t sdb, void *stream) {
    return gradients(M, N, K, n, r, X, ldx, dY, lddy, H, dH, index, dA, ldda, sda, dB, lddb, sdb, true, stream);
}

int adapters_force_plan(int op, int config, int split_k) {
    if (op < ADAPTERS_OP_FORWARD || op > ADAPTERS_OP_INPUT_GRADIENT || config < -1 || split_k < 0 ||
        (config >= 0 && !gemm::fused_has(op == ADAPTERS_OP_FORWARD ? gemm::FUSED_ADAPT : gemm::FUSED_ADAPT_DX, config)))
        return GEMM_ERR_INVALID_VALUE;
    g_forced[op].config = config;
    g_forced[op].split = split_k;
    return GEMM_OK;
}

}  // extern "C"
