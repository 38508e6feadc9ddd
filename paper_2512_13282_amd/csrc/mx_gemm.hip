// mx_gemm.hip -- launches the products over block-scaled operands.
#include "families.h"
#include "mx_launch.h"

namespace gemm {

// The copies that MxCopy describes, both in one launch, for the launch is what the smaller ones cost.
__global__ __launch_bounds__(256) void mx_realign_kernel(MxCopy x, MxCopy y) {
    const int64_t x_total = x.rows * (x.pitch / 16), total = x_total + y.rows * (y.pitch / 16), step = int64_t(gridDim.x) * 256;
    for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < total; id += step) {
        const bool first = id < x_total;
        const int64_t at = first ? id : id - x_total, pieces = (first ? x.pitch : y.pitch) / 16;
        const int64_t r = (at | pieces) >> 32 == 0 ? uint32_t(at) / uint32_t(pieces) : at / pieces, c = at - r * pieces;
        const uint8_t *const p = first ? x.src + r * x.stride + 16 * c : y.src + r * y.stride + 16 * c;
        const int64_t left = (first ? x.used : y.used) - 16 * c;
        u32x4_t v{0u, 0u, 0u, 0u};
        if (left >= 16) {
            v = *reinterpret_cast<const u32x4_any_mx *>(p);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (e < left) v[e / 4] |= uint32_t(p[e]) << (8 * (e & 3));
        }
        *reinterpret_cast<u32x4_t *>(first ? x.dst + r * x.pitch + 16 * c : y.dst + r * y.pitch + 16 * c) = v;
    }
}

static bool mx_realign(const MxCopy &x, const MxCopy &y, hipStream_t stream) {
    const int64_t n = (x.rows * (x.pitch / 16) + y.rows * (y.pitch / 16) + 255) / 256;
    hipLaunchKernelGGL(mx_realign_kernel, dim3(unsigned(n < 65536 ? n : 65536)), dim3(256), 0, stream, x, y);
    return hipGetLastError() == hipSuccess;
}

int launch_mx_gemm(const MxArgs &a0, MxOp op, const MxPlan &plan, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    MxArgs a = a0;
    const MxConfig &c = kMxConfigs[plan.config];
    const bool decode = plan.config == kMxDecode || plan.config == kMxDecode48;
    const int64_t tm = decode ? 1 : (a.g.M + c.bm - 1) / c.bm, tn = (a.g.N + c.bn - 1) / c.bn;
    const int64_t grid = tm * tn * plan.split_k;
    a.g.k_chunk = plan.k_chunk;
    a.g.split_k = plan.split_k;
    a.g.tiles_m = int32_t(tm);
    a.g.tiles_n = int32_t(tn);
    a.g.group_m = 4;
    a.g.reduce_in_kernel = REDUCE_LAST_SLICE;

    // Scratch: the K slices' partial sums, and aligned copies of operands that need one (their rows are
    // no longer than kMxMostStride: mx_select).
    const int64_t a_rows = op == MX_DW ? a.g.K : a.g.M, a_used = (op == MX_DW ? a.g.M : a.g.K) * 2, a_row = mx_a_row(op, a.g.M, a.g.K);
    const int64_t b_rows = op == MX_FWD ? a.g.N : a.g.K, b_cols = op == MX_FWD ? a.g.K : a.g.N;
    const int64_t b_used = op == MX_DW ? b_cols : (b_cols + 1) / 2, b_row = mx_b_row(op, a.g.N, a.g.K);
    const int64_t s_used = (b_cols + kMxBlock - 1) / kMxBlock, s_row = (s_used + 15) / 16 * 16;
    const bool any_a = decode || (a.g.lda * 2 <= kMxMostStride && mx_direct_a(plan.config, a.g.M, a.g.N, a.g.K));
    const bool copy_a = !any_a && a.g.K > 0 && !mx_loadable(a.g.A, a.g.lda * 2);
    const bool copy_b = !decode && a.g.K > 0 && !mx_loadable(a.g.B, a.g.ldb);
    // The gradient kernel offsets scale rows in 32 bits too; any alignment will do.
    const bool copy_s = op != MX_FWD && a.g.K > 0 && a.ld_scales > kMxMostStride;
    // Partial sums: whole tiles (the decode kernel's: 16 rows), at least the planes that the separate reduction reads.
    const int64_t partial = a.g.split_k > 1 ? a.g.split_k * tm * tn * c.bm * c.bn * 4 : 0;
    const int64_t a_bytes = copy_a ? a_rows * a_row : 0, b_bytes = copy_b ? b_rows * b_row : 0;
    const int64_t s_bytes = copy_s ? b_rows * s_row : 0;
    WorkspaceHold hold;                  // over the copies, the product and its separate reduction
    if (partial + a_bytes + b_bytes + s_bytes > 0) {
        void *ws = nullptr;
        uint32_t *counters = nullptr;
        const size_t bytes = size_t(partial + a_bytes + b_bytes + s_bytes);
        int rc = acquire_workspace(stream_ptr, bytes, a.g.split_k > 1 ? tm * tn : 0, &ws, &counters, hold);
        if (rc == LAUNCH_NO_COUNTERS) {
            a.g.reduce_in_kernel = REDUCE_SEPARATE;     // the same sums in the same order
            rc = acquire_workspace(stream_ptr, bytes, 0, &ws, &counters, hold);
        }
        if (rc != LAUNCH_OK) return rc;
        a.g.workspace = ws;
        a.g.counters = counters;
        uint8_t *const copies = static_cast<uint8_t *>(ws) + partial;
        MxCopy x{}, y{};
        if (copy_a) {
            x = MxCopy{static_cast<const uint8_t *>(a.g.A), copies, a.g.lda * 2, a_used, a_row, a_rows};
            a.g.A = x.dst;
            a.g.lda = x.pitch / 2;
        }
        if (copy_b) {
            y = MxCopy{static_cast<const uint8_t *>(a.g.B), copies + a_bytes, a.g.ldb, b_used, b_row, b_rows};
            a.g.B = y.dst;
            a.g.ldb = y.pitch;
        }
        if ((copy_a || copy_b) && !mx_realign(x, y, stream)) return LAUNCH_HIP_ERROR;
        if (copy_s) {
            x = MxCopy{a.scales, copies + a_bytes + b_bytes, a.ld_scales, s_used, s_row, b_rows};
            a.scales = x.dst;
            a.ld_scales = x.pitch;
            if (!mx_realign(x, MxCopy{}, stream)) return LAUNCH_HIP_ERROR;
        }
    }
    hipError_t e = op == MX_FWD ? launch_mx_fwd(plan.config, a, grid, stream)
                 : op == MX_DX ? launch_mx_dx(plan.config, a, grid, stream) : launch_mx_dw(plan.config, a, grid, stream);
    if (e == hipSuccess && a.g.split_k > 1 && a.g.reduce_in_kernel == REDUCE_SEPARATE) {
        const int64_t blocks = (a.g.M * a.g.N + 255) / 256;
        e = launch_splitk_reduce<DT_BF16>(a.g, blocks < 8192 ? blocks : 8192, stream);
    }
    return e == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

}  // namespace gemm
