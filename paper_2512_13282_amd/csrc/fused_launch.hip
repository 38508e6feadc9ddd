// fused_launch.hip -- launches the fused products: copies of operands that need one, the adapters' first
// product, then the product itself.
#include "fused_launch.h"
#include "kern_adapters.h"
#include "mx_launch.h"

namespace gemm {

// Up to four operands of a product copied to aligned rows (mx_launch.h) in one launch.  Rows of bf16 may lie off dwords, where
// 16-byte loads are slow: dwords put together (load8_any).
struct FusedCopies {
    MxCopy job[4];
    int64_t end[4];                  // pieces of 16 bytes, this job's and those before it
};
__global__ __launch_bounds__(256) void fused_realign_kernel(FusedCopies c) {
    const int64_t step = int64_t(gridDim.x) * 256;
    for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < c.end[3]; id += step) {
        MxCopy j = c.job[0];
        int64_t at = id;
#pragma unroll
        for (int k = 1; k < 4; ++k)
            if (id >= c.end[k - 1]) {
                j = c.job[k];
                at = id - c.end[k - 1];
            }
        const int64_t pieces = j.pitch / 16;
        const int64_t r = (at | pieces) >> 32 == 0 ? uint32_t(at) / uint32_t(pieces) : at / pieces, col = 8 * (at - r * pieces);
        const uint16_t *const src = reinterpret_cast<const uint16_t *>(j.src + r * j.stride) + col;
        const int64_t left = j.used / 2 - col;
        *reinterpret_cast<u32x4_t *>(j.dst + r * j.pitch + 2 * col) = left >= 8 ? load8_any<true>(src) : load8_bf16(src, left);
    }
}

namespace {

bool realign(const MxCopy (&jobs)[4], int count, hipStream_t stream) {
    if (count == 0) return true;
    FusedCopies c{};
    int64_t end = 0;
    for (int k = 0; k < 4; ++k) {
        if (k < count) {
            c.job[k] = jobs[k];
            end += jobs[k].rows * (jobs[k].pitch / 16);
        }
        c.end[k] = end;
    }
    const int64_t blocks = (end + 255) / 256;
    hipLaunchKernelGGL(fused_realign_kernel, dim3(unsigned(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream, c);
    return hipGetLastError() == hipSuccess;
}

int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// Tokens and ranks of a block (in sixteens).
int shrink_rt(const ShrinkArgs &s) { return s.r <= 16 ? 1 : s.r <= 32 ? 2 : 4; }
int shrink_mt(const ShrinkArgs &s) { return s.M <= 64 ? 1 : s.M <= 512 || (shrink_rt(s) == 4 && !s.qt) ? 2 : 4; }

template <bool QT, int MT>
void queue_shrink_rows(const ShrinkArgs &s, dim3 grid, hipStream_t stream) {
    const int rt = shrink_rt(s);
    if (rt == 1) hipLaunchKernelGGL((adapters_shrink_kernel<QT, MT, 1, MT == 1 ? 16 : 8>), grid, dim3(MT == 1 ? 1024 : 512), 0, stream, s);
    else if (rt == 2) hipLaunchKernelGGL((adapters_shrink_kernel<QT, MT, 2, 8>), grid, dim3(512), 0, stream, s);
    else if constexpr (QT || MT < 4) hipLaunchKernelGGL((adapters_shrink_kernel<QT, MT, 4, 8>), grid, dim3(512), 0, stream, s);
}
template <bool QT>
hipError_t queue_shrink(const ShrinkArgs &s, hipStream_t stream) {
    const dim3 grid(unsigned(s.blocks * s.parts), unsigned(s.slices), unsigned(s.groups));
    const int mt = shrink_mt(s);
    if (mt == 1) queue_shrink_rows<QT, 1>(s, grid, stream);
    else if (mt == 2) queue_shrink_rows<QT, 2>(s, grid, stream);
    else queue_shrink_rows<QT, 4>(s, grid, stream);
    return hipGetLastError();
}

}  // namespace

int launch_fused_with(const FusedArgs &a0, FusedOp op, const FusedPlan &plan, const ShrinkArgs *shrink, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    FusedArgs a = a0;
    const FusedConfig &c = kFusedConfigs[plan.config];
    const int64_t cols = op == FUSED_GATED ? c.bn / 2 : c.bn;
    const bool any = fused_any_address(plan.config);
    const int64_t tm = (a.g.M + c.bm - 1) / c.bm * (op == FUSED_DW ? a.pairs : 1), tn = (a.g.N + cols - 1) / cols;
    const int64_t sliced = plan.split_k > 1 ? tm * tn - plan.whole : 0;
    int64_t grid = plan.whole + sliced * plan.split_k;
    a.g.k_chunk = plan.k_chunk;
    a.g.split_k = plan.split_k;
    a.whole = plan.whole;
    a.half = op == FUSED_DW ? int32_t((a.g.M + c.bm - 1) / c.bm) : INT32_MAX;
    if (c.low > 0) {
        const FusedTail t = fused_tail(op, a.pairs, a.g.M, a.g.N, plan);
        a.tail = FusedArgs::Tail{t.row, t.col, int32_t(t.tiles_m), int32_t(t.tiles_n), op == FUSED_DW ? int32_t(t.half) : INT32_MAX};
        grid += t.tiles;
        a.early = op == FUSED_GRAD && plan.whole > 128 ? int32_t(t.tiles < 128 ? t.tiles / 8 * 8 : 128) : 0;
    }
    a.g.tiles_m = int32_t(plan.tail_rows > 0 ? plan.tail_rows : tm);
    a.g.tiles_n = int32_t(plan.tail_cols > 0 ? plan.tail_cols : tn);
    a.g.group_m = 4;
    a.g.reduce_in_kernel = REDUCE_LAST_SLICE;

    // Scratch: the K slices' sums, the planes of h, and aligned copies of operands that need one.
    const int64_t partial = a.g.split_k > 1 ? sliced * plan.split_k * c.bm * c.bn * 4 : 0;
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
        copy[i] = !any && grid > 0 && o.rows > 0 && o.cols > 0 && !fused_loadable(*o.p, *o.ld, o.along_k, o.cols);
        if (copy[i]) copied += o.rows * up16(2 * o.cols);
    }
    // The kernels for few rows add h's planes up themselves; elsewhere and where the caller keeps h the slices meet in it.
    const bool sum_h = shrink != nullptr && shrink->slices > 1 && (shrink->h != nullptr || !fused_few_rows(plan.config));
    const bool own_h = shrink != nullptr && shrink->h == nullptr && sum_h;
    // The planes of h, or the slices' sums as registers hold them and h.
    int64_t planes = 0, h_at = 0;
    if (sum_h) {
        h_at = int64_t(shrink->blocks) * shrink->groups * shrink->slices * shrink_mt(*shrink) * shrink_rt(*shrink) * 1024;
        planes = h_at + (own_h ? up16(shrink->plane * 4) : 0);
    } else if (shrink != nullptr && (shrink->h == nullptr || shrink->slices > 1)) {
        planes = up16(shrink->slices * shrink->plane * 4);
    }
    const int64_t counted = sliced, h_counted = sum_h ? int64_t(shrink->blocks) * shrink->groups : 0;

    WorkspaceHold hold;                  // over the copies, the adapters' first product and the product
    if (partial + copied + planes > 0) {
        void *ws = nullptr;
        uint32_t *counters = nullptr;
        const int rc = acquire_counted(stream_ptr, size_t(partial + copied + planes), counted + h_counted, &ws, &counters, hold);
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
        if (!realign(jobs, n, stream)) return LAUNCH_HIP_ERROR;
    }
    if (shrink != nullptr) {
        ShrinkArgs s = *shrink;
        float *const own = reinterpret_cast<float *>(static_cast<uint8_t *>(a.g.workspace) + partial);
        s.out = planes > 0 ? own : s.h;
        if (own_h) s.h = own + h_at / 4;
        s.counters = sum_h ? a.g.counters + counted : nullptr;
        if ((s.qt ? queue_shrink<true>(s, stream) : queue_shrink<false>(s, stream)) != hipSuccess) return LAUNCH_HIP_ERROR;
        a.h = sum_h ? s.h : s.out;
        a.h_plane = s.plane;
        a.planes = sum_h ? 1 : s.slices;
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

// Eight columns of a row to a thread, at any address and stride.  Bound by memory: ten bytes an element (2048 x 11008: 38.9 us,
// 5.8 TB/s).
__global__ __launch_bounds__(256) void gated_bwd_kernel(GatedBwdArgs a) {
    const int64_t pieces = (a.N + 7) / 8, total = a.M * pieces;
    with_act(a.act, [&](auto act) __attribute__((always_inline)) {
        constexpr int ACT = decltype(act)::value;
        for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < total; id += int64_t(gridDim.x) * 256) {
            const int64_t row = (id | pieces) >> 32 == 0 ? uint32_t(id) / uint32_t(pieces) : id / pieces, col = 8 * (id - row * pieces), left = a.N - col;
            const u32x4_t d = load8_bf16(static_cast<const uint16_t *>(a.dH) + row * a.lddh + col, left);
            const u32x4_t g = load8_bf16(static_cast<const uint16_t *>(a.G) + row * a.ldg + col, left);
            const u32x4_t u = load8_bf16(static_cast<const uint16_t *>(a.U) + row * a.ldu + col, left);
            float dg[8], du[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                auto value = [&](const u32x4_t &v) __attribute__((always_inline)) { return bf16_to_f32((v[e / 2] >> (16 * (e & 1))) & 0xffffu); };
                float val, slope;
                act_both<ACT>(value(g), val, slope);
                dg[e] = value(d) * value(u) * slope;
                du[e] = value(d) * val;
            }
            uint16_t *const og = static_cast<uint16_t *>(a.dG) + row * a.lddg + col, *const ou = static_cast<uint16_t *>(a.dU) + row * a.lddu + col;
            store4_bf16(og, left, pack_bf16(dg[0], dg[1]), pack_bf16(dg[2], dg[3]));
            store4_bf16(ou, left, pack_bf16(du[0], du[1]), pack_bf16(du[2], du[3]));
            store4_bf16(og + 4, left - 4, pack_bf16(dg[4], dg[5]), pack_bf16(dg[6], dg[7]));
            store4_bf16(ou + 4, left - 4, pack_bf16(du[4], du[5]), pack_bf16(du[6], du[7]));
        }
    });
}

int launch_gated_bwd(const GatedBwdArgs &a, void *stream) {
    const int64_t blocks = (a.M * ((a.N + 7) / 8) + 255) / 256;
    hipLaunchKernelGGL(gated_bwd_kernel, dim3(unsigned(blocks < 16384 ? blocks : 16384)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return hipGetLastError() == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

int launch_fused(const FusedArgs &a, FusedOp op, const FusedPlan &plan, void *stream) { return launch_fused_with(a, op, plan, nullptr, stream); }

int launch_adapters(const FusedArgs &a, FusedOp op, const FusedPlan &plan, const ShrinkArgs &s0, void *stream) {
    if (s0.r == 0 || (s0.n == 0 && s0.h == nullptr)) return launch_fused_with(a, op, plan, nullptr, stream);
    ShrinkArgs s = s0;
    if (s.n == 0) s.L = 0;               // zeros
    // Slices of at least 512 of L until every compute unit has a workgroup; then the adapters of a block apart, of which
    // few tokens have one each and many most often one.
    s.blocks = int32_t((s.M + 16 * shrink_mt(s) - 1) / (16 * shrink_mt(s)));
    s.groups = (s.r + 16 * shrink_rt(s) - 1) / (16 * shrink_rt(s));
    const int64_t wanted = 256 / (int64_t(s.blocks) * s.groups), most = (s.L + 511) / 512;
    int64_t slices = wanted < most ? wanted : most;
    if (slices > 8) slices = 8;
    if (slices < 1) slices = 1;
    int64_t parts = 2 * wanted / slices;
    if (parts > s.M) parts = s.M;
    if (parts > s.n) parts = s.n;
    if (parts > 16) parts = 16;
    if (parts < 1) parts = 1;
    s.parts = int32_t(parts);
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
