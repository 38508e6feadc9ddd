// mx_api.cpp -- the C ABI entry points of the block-scaled products (host side): argument
// checks before any HIP call, then the launch.
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "../../include/mx_mi355x.h"
#include "mx.h"
#include "region.h"

namespace {

using gemm::Region;
using gemm::region;

int64_t code_bytes(int64_t cols, int bits) { return bits == 4 ? cols / 2 + cols % 2 : cols; }
int64_t blocks(int64_t cols) { return cols / gemm::kMxBlock + (cols % gemm::kMxBlock != 0); }

int status(int launched) {
    switch (launched) {
        case gemm::LAUNCH_OK: return GEMM_OK;
        case gemm::LAUNCH_NO_MEMORY: return GEMM_ERR_NO_MEMORY;
        default: return GEMM_ERR_HIP;
    }
}

int convert(bool pack, int bits, int64_t rows, int64_t cols, const void *x, int64_t ldx, const void *codes, int64_t ldq,
            const uint8_t *scales, int64_t lds, void *stream) {
    if (rows < 0 || cols < 0) return GEMM_ERR_INVALID_VALUE;
    const Region rx = region(x, rows, cols, ldx, 2);
    const Region rq = region(codes, rows, code_bytes(cols, bits), ldq, 1);
    const Region rs = region(scales, rows, blocks(cols), lds, 1);
    if (!rx.valid() || !rq.valid() || !rs.valid()) return GEMM_ERR_INVALID_VALUE;
    if (rx.overlaps(rq) || rx.overlaps(rs) || (pack && rq.overlaps(rs))) return GEMM_ERR_INVALID_VALUE;
    if (rows == 0 || cols == 0) return GEMM_OK;
    const gemm::MxMatrixArgs a{rows, cols, const_cast<void *>(x), ldx, const_cast<void *>(codes), ldq,
                               const_cast<uint8_t *>(scales), lds};
    return status(pack ? gemm::launch_mx_pack(a, bits, stream) : gemm::launch_mx_unpack(a, bits, stream));
}

struct Forced {
    std::atomic<int32_t> config{-1}, split{0};
};
Forced g_forced[3];

// The plans of this thread's latest shapes: choosing one evaluates a hundred or so.
struct CachedPlan {
    int64_t M, N, K, copied_a, copied_b;   // M = 0: empty
    int32_t op;
    gemm::MxPlan plan;
};
thread_local CachedPlan t_plans[64];

int plan_for(gemm::MxOp op, int64_t M, int64_t N, int64_t K, int64_t copied_a, int64_t copied_b, gemm::MxPlan *plan) {
    constexpr int64_t kMost = INT32_MAX - 4096;      // 32-bit indices, up to the end of a tile or a stage
    if (M > kMost || N > kMost || K > kMost) return GEMM_ERR_UNSUPPORTED;
    const int32_t config = g_forced[op].config, split = g_forced[op].split;
    if (config >= 0 || split > 0)
        return gemm::mx_select(op, M, N, K, copied_a, copied_b, config, split, plan) ? GEMM_OK : GEMM_ERR_UNSUPPORTED;
    const uint64_t h = (uint64_t(M) * 0x9E3779B97F4A7C15u ^ uint64_t(N) * 0xC2B2AE3D27D4EB4Fu ^ uint64_t(K) * 0x165667B19E3779F9u) + uint64_t(op);
    CachedPlan &c = t_plans[(h ^ (h >> 32)) % 64];
    if (c.M != M || c.N != N || c.K != K || c.copied_a != copied_a || c.copied_b != copied_b || c.op != op) {
        gemm::MxPlan p;
        if (!gemm::mx_select(op, M, N, K, copied_a, copied_b, -1, 0, &p)) return GEMM_ERR_UNSUPPORTED;
        c = CachedPlan{M, N, K, copied_a, copied_b, op, p};
    }
    *plan = c.plan;
    return GEMM_OK;
}

int product(gemm::MxOp op, int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda, const void *codes,
            int64_t ldq, const uint8_t *scales, int64_t lds, void *C, int64_t ldc, bool bf16_out, void *stream) {
    if (M < 0 || N < 0 || K < 0) return GEMM_ERR_INVALID_VALUE;
    const int bits = op == gemm::MX_DW ? 8 : 4;
    const Region ra = op == gemm::MX_DW ? region(A, K, M, lda, 2) : region(A, M, K, lda, 2);
    const int64_t b_rows = op == gemm::MX_FWD ? N : K, b_cols = op == gemm::MX_FWD ? K : N;
    const Region rq = region(codes, b_rows, code_bytes(b_cols, bits), ldq, 1);
    const Region rs = region(scales, b_rows, blocks(b_cols), lds, 1);
    const Region rc = region(C, M, N, ldc, bf16_out ? 2 : 4);
    if (!ra.valid() || !rq.valid() || !rs.valid() || !rc.valid()) return GEMM_ERR_INVALID_VALUE;
    if (rc.overlaps(ra) || rc.overlaps(rq) || rc.overlaps(rs)) return GEMM_ERR_INVALID_VALUE;
    if (M == 0 || N == 0) return GEMM_OK;
    gemm::MxPlan plan;
    // What a tile kernel would have copied first.
    const int64_t copied_a = K == 0 || gemm::mx_loadable(A, ra.stride) ? 0 : ra.rows * ra.used;
    const int64_t copied_b = K == 0 || gemm::mx_loadable(codes, ldq) ? 0 : rq.rows * rq.used;
    const int planned = plan_for(op, M, N, K, copied_a, copied_b, &plan);
    if (planned != GEMM_OK) return planned;
    gemm::MxArgs a{};
    a.g.dtype = 1;      // bf16 operands on the MFMAs
    a.g.A = A;
    a.g.B = codes;
    a.g.C = C;
    a.g.M = M; a.g.N = N; a.g.K = K;
    a.g.lda = lda; a.g.ldb = ldq; a.g.ldc = ldc;
    a.g.epilogue = bf16_out ? gemm::EPI_BF16 : gemm::EPI_NONE;
    a.scales = scales;
    a.ld_scales = lds;
    try {
        return status(gemm::launch_mx_gemm(a, op, plan, stream));
    } catch (...) {      // the workspace table's own memory
        return GEMM_ERR_NO_MEMORY;
    }
}

}  // namespace

extern "C" {

int mx_pack4(int64_t rows, int64_t cols, const uint16_t *X, int64_t ldx, uint8_t *codes, int64_t ldq, uint8_t *scales,
             int64_t lds, void *stream) {
    return convert(true, 4, rows, cols, X, ldx, codes, ldq, scales, lds, stream);
}

int mx_pack8(int64_t rows, int64_t cols, const uint16_t *X, int64_t ldx, int8_t *codes, int64_t ldq, uint8_t *scales,
             int64_t lds, void *stream) {
    return convert(true, 8, rows, cols, X, ldx, codes, ldq, scales, lds, stream);
}

int mx_unpack4(int64_t rows, int64_t cols, const uint8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
               uint16_t *X, int64_t ldx, void *stream) {
    return convert(false, 4, rows, cols, X, ldx, codes, ldq, scales, lds, stream);
}

int mx_unpack8(int64_t rows, int64_t cols, const int8_t *codes, int64_t ldq, const uint8_t *scales, int64_t lds,
               uint16_t *X, int64_t ldx, void *stream) {
    return convert(false, 8, rows, cols, X, ldx, codes, ldq, scales, lds, stream);
}

int mx_gemm_bf16_mx4_f32_bt(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda, const uint8_t *codes,
                            int64_t ldq, const uint8_t *scales, int64_t lds, float *C, int64_t ldc, void *stream) {
    return product(gemm::MX_FWD, M, N, K, A, lda, codes, ldq, scales, lds, C, ldc, false, stream);
}

int mx_gemm_bf16_mx4_bf16_bt(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda, const uint8_t *codes,
                             int64_t ldq, const uint8_t *scales, int64_t lds, uint16_t *C, int64_t ldc, void *stream) {
    return product(gemm::MX_FWD, M, N, K, A, lda, codes, ldq, scales, lds, C, ldc, true, stream);
}

int mx_gemm_bf16_mx4_f32(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda, const uint8_t *codes,
                         int64_t ldq, const uint8_t *scales, int64_t lds, float *C, int64_t ldc, void *stream) {
    return product(gemm::MX_DX, M, N, K, A, lda, codes, ldq, scales, lds, C, ldc, false, stream);
}

int mx_gemm_bf16_mx4_bf16(int64_t M, int64_t N, int64_t K, const uint16_t *A, int64_t lda, const uint8_t *codes,
                          int64_t ldq, const uint8_t *scales, int64_t lds, uint16_t *C, int64_t ldc, void *stream) {
    return product(gemm::MX_DX, M, N, K, A, lda, codes, ldq, scales, lds, C, ldc, true, stream);
}

int mx_gemm_bf16_mx8_f32_at(int64_t M, int64_t N, int64_t K, const uint16_t *At, int64_t ldat, const int8_t *codes,
                            int64_t ldq, const uint8_t *scales, int64_t lds, float *C, int64_t ldc, void *stream) {
    return product(gemm::MX_DW, M, N, K, At, ldat, codes, ldq, scales, lds, C, ldc, false, stream);
}

int mx_gemm_bf16_mx8_bf16_at(int64_t M, int64_t N, int64_t K, const uint16_t *At, int64_t ldat, const int8_t *codes,
                             int64_t ldq, const uint8_t *scales, int64_t lds, uint16_t *C, int64_t ldc, void *stream) {
    return product(gemm::MX_DW, M, N, K, At, ldat, codes, ldq, scales, lds, C, ldc, true, stream);
}

int mx_plan(int op, int64_t M, int64_t N, int64_t K, mx_plan_info *out) {
    if (out == nullptr || op < MX_OP_FORWARD || op > MX_OP_WEIGHT_GRADIENT || M < 0 || N < 0 || K < 0)
        return GEMM_ERR_INVALID_VALUE;
    memset(out, 0, sizeof(*out));
    out->config = -1;
    if (M == 0 || N == 0) return GEMM_OK;
    gemm::MxPlan plan;
    // Rows on 16 bytes, but of what is longer than the tile kernels can step over.
    const gemm::MxOp o = gemm::MxOp(op);
    const bool sizes = M <= INT32_MAX && N <= INT32_MAX && K <= INT32_MAX;       // else plan_for refuses
    const int64_t a_row = sizes ? gemm::mx_a_row(o, M, K) : 0, b_row = sizes ? gemm::mx_b_row(o, N, K) : 0;
    const int rc = plan_for(o, M, N, K, a_row > gemm::kMxMostStride ? a_row * (o == gemm::MX_DW ? K : M) : 0,
                            b_row > gemm::kMxMostStride ? b_row * (o == gemm::MX_FWD ? N : K) : 0, &plan);
    if (rc != GEMM_OK) return rc;
    const gemm::MxConfig &c = gemm::kMxConfigs[plan.config];
    out->config = plan.config;
    out->bm = c.bm;
    out->bn = c.bn;
    out->split_k = plan.split_k;
    out->k_chunk = plan.k_chunk;
    strncpy(out->name, c.name, sizeof(out->name) - 1);
    return GEMM_OK;
}

int mx_force_plan(int op, int config, int split_k) {
    if (op < MX_OP_FORWARD || op > MX_OP_WEIGHT_GRADIENT || config < -1 || config >= gemm::kMxNumConfigs || split_k < 0 ||
        (config >= 0 && gemm::kMxConfigs[config].op != op))
        return GEMM_ERR_INVALID_VALUE;
    g_forced[op].config = config;
    g_forced[op].split = split_k;
    return GEMM_OK;
}

}  // extern "C"
