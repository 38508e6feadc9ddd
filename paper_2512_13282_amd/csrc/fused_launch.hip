// fused_launch.hip -- launches the fused products: copies of operands that need one, the adapters' first
// product, then the product itself.
#include "fused_launch.h"
#include "kern_adapters.h"
#include "mx_launch.h"

namespace gemm {

namespace {

int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

template <bool QT>
hipError_t queue_shrink(const ShrinkArgs &s, hipStream_t stream) {
    const int rt = s.r <= 16 ? 1 : s.r <= 32 ? 2 : 4;
    const dim3 grid(unsigned((s.M + 15) / 16), unsigned(s.slices), unsigned((s.r + 16 * rt - 1) / (16 * rt)));
    if (rt == 1) hipLaunchKernelGGL((adapters_shrink_kernel<QT, 1, 1, 8>), grid, dim3(512), 0, stream, s);
    else if (rt == 2) hipLaunchKernelGGL((adapters_shrink_kernel<QT, 1, 2, 8>), grid, dim3(512), 0, stream, s);
    else hipLaunchKernelGGL((adapters_shrink_kernel<QT, 1, 4, 8>), grid, dim3(512), 0, stream, s);
    return hipGetLastError();
}

}  // namespace

int launch_fused_with(const FusedArgs &a0, FusedOp op, const FusedPlan &plan, const ShrinkArgs *shrink, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    FusedArgs a = a0;
    const FusedConfig &c = kFusedConfigs[plan.config];
    const int64_t cols = op == FUSED_GATED ? c.bn / 2 : c.bn;
    const int64_t tm = (a.g.M + c.bm - 1) / c.bm * (op == FUSED_DW ? a.pairs : 1), tn = (a.g.N + cols - 1) / cols;
    const int64_t grid = tm * tn * plan.split_k;
    a.g.k_chunk = plan.k_chunk;
    a.g.split_k = plan.split_k;
    a.g.tiles_m = int32_t(tm);
    a.g.tiles_n = int32_t(tn);
    a.g.group_m = 4;
    a.g.reduce_in_kernel = REDUCE_LAST_SLICE;

    // Scratch: the K slices' sums, the planes of h, and aligned copies of operands that need one.
    const int64_t partial = a.g.split_k > 1 ? grid * c.bm * c.bn * 4 : 0;
    const bool at = op == FUSED_DW, bt = op == FUSED_GATED || op == FUSED_ADAPT;
    const int64_t a_rows = at ? a.g.K : a.g.M, a_cols = at ? a.g.M : a.g.K;
    const int64_t b_rows = bt ? a.g.N : a.g.K, b_cols = bt ? a.g.K : a.g.N;
    struct Operand { const void **p; int64_t *ld; int64_t rows, cols; bool along_k; };
    const Operand operands[4] = {{&a.g.A, &a.g.lda, a_rows, a_cols, !at}, {&a.g.B, &a.g.ldb, b_rows, b_cols, bt},
                                 {&a.A2, &a.lda2, a.A2 != nullptr ? a_rows : 0, a_cols, !at},
                                 {&a.B2, &a.ldb2, a.B2 != nullptr ? b_rows : 0, b_cols, bt}};
    int64_t copied = 0;
    bool copy[4];
    for (int i = 0; i < 4; ++i) {
        const Operand &o = operands[i];
        copy[i] = o.rows > 0 && o.cols > 0 && !fused_loadable(*o.p, *o.ld, o.along_k, o.cols);
        if (copy[i]) copied += o.rows * up16(2 * o.cols);
    }
    const int64_t planes = shrink != nullptr && (shrink->h == nullptr || shrink->slices > 1) ? up16(shrink->slices * shrink->plane * 4) : 0;

    WorkspaceHold hold;                  // over the copies, the adapters' first product and the product
    if (partial + copied + planes > 0) {
        void *ws = nullptr;
        uint32_t *counters = nullptr;
        const int rc = acquire_counted(stream_ptr, size_t(partial + copied + planes), a.g.split_k > 1 ? tm * tn : 0, &ws, &counters, hold);
        if (rc != LAUNCH_OK) return rc;
        a.g.workspace = ws;
        a.g.counters = counters;
        uint8_t *at_copy = static_cast<uint8_t *>(ws) + partial + planes;
        MxCopy jobs[4];
        int n = 0;
        for (int i = 0; i < 4; ++i) {
            if (!copy[i]) continue;
            const Operand &o = operands[i];
            jobs[n] = MxCopy{static_cast<const uint8_t *>(*o.p), at_copy, *o.ld * 2, o.cols * 2, up16(2 * o.cols), o.rows};
            at_copy += o.rows * jobs[n].pitch;
            *o.p = jobs[n].dst;
            *o.ld = jobs[n].pitch / 2;
            ++n;
        }
        for (int i = 0; i < n; i += 2)
            if (!mx_realign(jobs[i], i + 1 < n ? jobs[i + 1] : MxCopy{}, stream)) return LAUNCH_HIP_ERROR;
    }
    if (shrink != nullptr) {
        ShrinkArgs s = *shrink;
        float *const own = reinterpret_cast<float *>(static_cast<uint8_t *>(a.g.workspace) + partial);
        s.out = s.h != nullptr && s.slices == 1 ? s.h : own;
        if ((s.qt ? queue_shrink<true>(s, stream) : queue_shrink<false>(s, stream)) != hipSuccess) return LAUNCH_HIP_ERROR;
        a.h = s.out;
        a.h_plane = s.plane;
        a.planes = s.slices;
        if (s.h != nullptr && s.slices > 1) {
            const int64_t total = s.M * s.r, blocks = (total + 255) / 256;
            hipLaunchKernelGGL(adapters_sum_kernel, dim3(unsigned(blocks < 1024 ? blocks : 1024)), dim3(256), 0, stream, own, s.plane,
                               s.slices, s.h, total);
            if (hipGetLastError() != hipSuccess) return LAUNCH_HIP_ERROR;
            a.h = s.h;
            a.planes = 1;
        }
    }
    if (grid == 0) return LAUNCH_OK;      // h alone
    hipError_t e = hipErrorInvalidValue;
    switch (op) {
        case FUSED_GATED: e = launch_fused_gated(plan.config, a, grid, stream); break;
        case FUSED_GRAD: e = launch_fused_grad(plan.config, a, grid, stream); break;
        case FUSED_DX: e = launch_fused_dx(plan.config, a, grid, stream); break;
        case FUSED_DW: e = launch_fused_dw(plan.config, a, grid, stream); break;
        case FUSED_ADAPT: e = launch_fused_adapt(plan.config, a, grid, stream); break;
        case FUSED_ADAPT_DX: e = launch_fused_adapt_dx(plan.config, a, grid, stream); break;
        default: break;
    }
    return e == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

int launch_fused(const FusedArgs &a, FusedOp op, const FusedPlan &plan, void *stream) { return launch_fused_with(a, op, plan, nullptr, stream); }

int launch_adapters(const FusedArgs &a, FusedOp op, const FusedPlan &plan, const ShrinkArgs &s0, void *stream) {
    if (s0.r == 0 || (s0.n == 0 && s0.h == nullptr)) return launch_fused_with(a, op, plan, nullptr, stream);
    ShrinkArgs s = s0;
    if (s.n == 0) s.L = 0;               // zeros
    // Slices of at least 256 until the compute units have a workgroup each; every reader of h adds the planes up.
    const int rt = s.r <= 16 ? 1 : s.r <= 32 ? 2 : 4;
    const int64_t groups = (s.M + 15) / 16 * ((s.r + 16 * rt - 1) / (16 * rt));
    int64_t slices = 256 / groups, most = (s.L + 255) / 256;
    if (slices > most) slices = most;
    if (slices > 8) slices = 8;
    if (slices < 1) slices = 1;
    s.chunk = s.L > 0 ? ((s.L + slices - 1) / slices + 31) / 32 * 32 : 32;
    s.slices = int32_t(s.L > 0 ? (s.L + s.chunk - 1) / s.chunk : 1);
    s.plane = s.M * s.r;
    return launch_fused_with(a, op, plan, &s, stream);
}

int launch_adapters_dw(const AdapterDwArgs &a, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    const int rt = a.r <= 16 ? 1 : a.r <= 32 ? 2 : 4;
    const dim3 grid(unsigned(a.side[0].blocks + a.side[1].blocks), unsigned(a.n), unsigned((a.r + 16 * rt - 1) / (16 * rt)));
    if (rt == 1) hipLaunchKernelGGL(adapters_dw_kernel<1>, grid, dim3(256), 0, stream, a);
    else if (rt == 2) hipLaunchKernelGGL(adapters_dw_kernel<2>, grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(adapters_dw_kernel<4>, grid, dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

}  // namespace gemm
