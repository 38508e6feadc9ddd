// kern_fused_tile.h -- the fused products on output tiles of up to 128 x 256.
#pragma once

#include "fused_common.h"
#include "fused_expand.h"

namespace gemm {

template <int OP> struct FusedLayout {
    static constexpr bool AT = OP == FUSED_DW;                               // A stored K x M
    static constexpr bool BT = OP == FUSED_GATED || OP == FUSED_ADAPT;       // B stored N x K
    static constexpr bool EXPAND = OP == FUSED_ADAPT || OP == FUSED_ADAPT_DX;
    static constexpr int HALVES = OP == FUSED_GATED ? 2 : 1;                 // column halves that are the same columns
};

// The epilogue of every fused product: whole sums in registers, tile row r0 and column c0 of the wave.
// tm: the tile's row of tiles (DW: the second matrix's follow the first's).
template <int OP, int THREADS, int HALF, int TM, int TN>
__device__ __forceinline__ void store_fused(const FusedArgs &a, f32x16_t (&acc)[TM][TN], int which, int64_t r0, int64_t c0, int lane) {
    if constexpr (OP == FUSED_GATED) {
        store_gated(a, acc, r0, c0, lane);
    } else if constexpr (OP == FUSED_GRAD) {
        with_act(a.act, [&](auto act) __attribute__((always_inline)) { store_grad_as<decltype(act)::value, HALF>(a, acc, r0, c0, lane); });
    } else {
        KernelArgs g = a.g;
        if (OP == FUSED_DW && which) {
            g.C = a.C2;
            g.ldc = a.ldc2;
        }
        store_plain<THREADS / 64, HALF>(g, acc, r0, c0, lane);
    }
}

// ---------------------------------------------------------------------------
// BM x BN output tile, WM x WN waves with BM / WM x 64 sums each: one 32-column fragment in each half of the
// tile's columns.  Both operands go straight into NS LDS stages of 64 k, and each iteration waits only for its own
// stage (gemm_lds_kernel's three-stage form says how); stages past the end load zeros.
//
// What lies along k (A, and B given N x K) sits in rows of 128 bytes, chunks swizzled by swz; what lies
// across it (B given K x N, and A given K x M) in 64 rows of k, read back transposed.  GATED: the halves are the same
// columns of two weights, so a lane holds g and u of the same outputs.  DX: the stages of the
// second product follow those of the first.  DW: the tiles of the second A follow those of the first.
//
// Serves what the larger tiles would leave compute units idle for.  Bound by the load path (about 50 GB/s a compute unit):
// dx 96 x 4096 x 2 . 11008 in eight slices 45.9 us with 128 x 128 tiles (eight waves, one workgroup to a unit), 51.9 with
// 64 x 128 in four slices (four waves, two to a unit), which read each weight twice there; 56 with 128 x 256.
// ---------------------------------------------------------------------------
template <int OP, int BM, int BN, int WM, int WN, int WAVES_PER_EU, int NS>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * WM * WN, 64 * WM * WN),
                          amdgpu_waves_per_eu(WAVES_PER_EU, WAVES_PER_EU)))
void fused_tile_kernel(FusedArgs a) {
    using L = FusedLayout<OP>;
    constexpr int WAVES = WM * WN, THREADS = 64 * WAVES, BK = 64;
    constexpr int TM = BM / WM / 32, TN = 2, HALF = BN / 2;
    static_assert(BN == 64 * WN && BM % (32 * WM) == 0, "a wave's tile");
    constexpr int A_STAGE = BM * 128, B_STAGE = BN * 128;
    constexpr int A_PITCH = L::AT ? BM * 2 : 128, B_PITCH = L::BT ? 128 : BN * 2;
    constexpr int A_CPR = A_PITCH / 16, B_CPR = B_PITCH / 16;
    constexpr int A_INSTR = A_STAGE / 1024 / WAVES, B_INSTR = B_STAGE / 1024 / WAVES;
    constexpr int LPS = A_INSTR + B_INSTR;
    static_assert(A_INSTR >= 1 && A_INSTR * 1024 * WAVES == A_STAGE, "A stage split");
    static_assert(B_INSTR >= 1 && B_INSTR * 1024 * WAVES == B_STAGE, "B stage split");
    static_assert(!L::BT || HALF % (8 * WAVES) == 0, "a load's rows belong to one half");
    static_assert(NS >= 3 && (NS - 1) * LPS < 64, "loads in flight must fit vmcnt");

    __shared__ __attribute__((aligned(1024))) uint8_t lds[NS][A_STAGE + B_STAGE];

    const int tid = int(threadIdx.x), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave_m = wave / WN, wave_n = wave % WN;
    constexpr int COLS = BN / L::HALVES;                         // output columns of a tile
    const int64_t M = a.g.M, N = a.g.N, K = a.g.K;
    const int one = int((K + BK - 1) / BK);                     // stages of one product
    const FusedWork work = fused_work<BM, 0, COLS>(a, OP == FUSED_DX ? 2 * one : one);
    const int64_t m0 = work.m0, n0 = work.n0;
    const int which = work.which, first = work.first, nk = work.count;
    const uint8_t *const a_src = static_cast<const uint8_t *>(which ? a.A2 : a.g.A);
    const int64_t lda_b = (which ? a.lda2 : a.g.lda) * 2, lda2_b = a.lda2 * 2;
    const int64_t ldb_b = a.g.ldb * 2, ldb2_b = a.ldb2 * 2;
    const int64_t rows_valid = M - m0 < BM ? M - m0 : BM;

    // ---- where this lane's pieces come from; the second operands' rows have strides of their own ----
    uint32_t a_voff[A_INSTR], a2_voff[A_INSTR];
    int a_chunk[A_INSTR];
#pragma unroll
    for (int i = 0; i < A_INSTR; ++i) {
        if constexpr (L::AT) {
            const int row = (i * WAVES + wave) * (1024 / A_PITCH) + lane / A_CPR;
            const int c = (lane % A_CPR) ^ ring_bswz<DT_BF16, A_CPR>(row);
            a_chunk[i] = 0;
            a_voff[i] = m0 + 8 * c < M ? uint32_t(row * lda_b + c * 16) : kOOB;
        } else {
            const int row = (i * WAVES + wave) * 8 + (lane >> 3);
            a_chunk[i] = swz(lane & 7, row);
            a_voff[i] = uint32_t(row * lda_b + a_chunk[i] * 16);
            a2_voff[i] = uint32_t(row * lda2_b + a_chunk[i] * 16);
        }
    }
    uint32_t b_voff[B_INSTR], b2_voff[B_INSTR];
    int b_chunk[B_INSTR];
#pragma unroll
    for (int i = 0; i < B_INSTR; ++i) {
        if constexpr (L::BT) {
            const int row = (i * WAVES + wave) * 8 + (lane >> 3);
            const bool up = L::HALVES == 2 && i * WAVES * 8 >= HALF;
            b_chunk[i] = swz(lane & 7, row);
            b_voff[i] = up ? uint32_t((row - HALF) * ldb2_b + b_chunk[i] * 16) : uint32_t(row * ldb_b + b_chunk[i] * 16);
        } else {
            const int row = (i * WAVES + wave) * (1024 / B_PITCH) + lane / B_CPR;
            const int c = (lane % B_CPR) ^ ring_bswz<DT_BF16, B_CPR>(row);
            b_chunk[i] = 0;
            b_voff[i] = n0 + 8 * c < N ? uint32_t(row * ldb_b + c * 16) : kOOB;
            b2_voff[i] = n0 + 8 * c < N ? uint32_t(row * ldb2_b + c * 16) : kOOB;
        }
    }
    const int64_t cols_valid = N - n0 < COLS ? N - n0 : COLS;     // rows of B given N x K

    auto load_stage = [&](int kt, auto buf_c) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_c)::value;
        int t = first + kt;
        const bool live = kt < nk;
        const bool second = OP == FUSED_DX && t >= one;
        if (second) t -= one;
        const int64_t k = int64_t(t) * BK;
        const int rem = live ? int(K - k < BK ? K - k : BK) : 0;
        const uint32_t dst = lds_addr(lds[BUF]) + uint32_t(wave) * 1024u;
        {
            const uint8_t *const src = second ? static_cast<const uint8_t *>(a.A2) : a_src;
            const int64_t ld = second ? lda2_b : lda_b;
            const uint8_t *const base = L::AT ? src + k * ld + m0 * 2 : src + m0 * ld + k * 2;
            const int64_t bytes = L::AT ? rem * ld : (rem > 0 ? rows_valid * ld : 0);
            const i32x4_t r = ring_rsrc(uniform(base), uniform(uint32_t(bytes)));
#pragma unroll
            for (int i = 0; i < A_INSTR; ++i) {
                const uint32_t off = !L::AT && second ? a2_voff[i] : a_voff[i];
                ring_load16(r, dst + i * (WAVES * 1024), L::AT || a_chunk[i] * 8 < rem ? off : kOOB);
            }
        }
        if constexpr (L::BT) {
            const i32x4_t r = ring_rsrc(uniform(static_cast<const uint8_t *>(a.g.B) + n0 * ldb_b + k * 2),
                                        uniform(uint32_t(rem > 0 ? cols_valid * ldb_b : 0)));
            const i32x4_t r2 = L::HALVES == 2 ? ring_rsrc(uniform(static_cast<const uint8_t *>(a.B2) + n0 * ldb2_b + k * 2),
                                                          uniform(uint32_t(rem > 0 ? cols_valid * ldb2_b : 0))) : r;
#pragma unroll
            for (int i = 0; i < B_INSTR; ++i)
                ring_load16(L::HALVES == 2 && i * WAVES * 8 >= HALF ? r2 : r, dst + A_STAGE + i * (WAVES * 1024),
                            b_chunk[i] * 8 < rem ? b_voff[i] : kOOB);
        } else {
            const int64_t ld = second ? ldb2_b : ldb_b;
            const uint8_t *const src = static_cast<const uint8_t *>(second ? a.B2 : a.g.B);
            const i32x4_t r = ring_rsrc(uniform(src + k * ld + n0 * 2), uniform(uint32_t(rem * ld)));
#pragma unroll
            for (int i = 0; i < B_INSTR; ++i) ring_load16(r, dst + A_STAGE + i * (WAVES * 1024), second ? b2_voff[i] : b_voff[i]);
        }
    };

    // ---- fragment offsets ----
    const int frag_row = lane & 31, frag_half = lane >> 5;
    const int wrow0 = wave_m * (BM / WM), wcol0 = wave_n * 32;
    const int r0 = wrow0 + frag_row, rb0 = wcol0 + frag_row;
    int a_fo[4], bt_fo[4];                                       // along k: k-step st of the wave's first 32 rows
#pragma unroll
    for (int st = 0; st < 4; ++st) {
        a_fo[st] = r0 * 128 + 16 * swz(2 * st + frag_half, r0);
        bt_fo[st] = rb0 * 128 + 16 * swz(2 * st + frag_half, rb0);
    }
    // Across k: transpose reads, as in gemm_lds_kernel.
    const int grp = lane >> 4, g16 = lane & 15;
    const int tr_row = g16 >> 2, tr_colb = (g16 & 3) * 8 + (grp & 1) * 32, tr_k = (grp >> 1) * 8 + tr_row;
    int at_fo[TM], b_fo[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int colb = (wrow0 + i * 32) * 2 + tr_colb;
        at_fo[i] = tr_k * A_PITCH + (((colb >> 4) ^ ring_bswz<DT_BF16, A_CPR>(tr_row)) << 4) + (colb & 15);
    }
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int colb = (wcol0 + j * HALF) * 2 + tr_colb;
        b_fo[j] = tr_k * B_PITCH + (((colb >> 4) ^ ring_bswz<DT_BF16, B_CPR>(tr_row)) << 4) + (colb & 15);
    }

    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};

    auto iteration = [&](int kt, auto buf_c) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_c)::value;
        ring_barrier<(NS - 2) * LPS>();
        load_stage(kt + NS - 1, std::integral_constant<int, (BUF + NS - 1) % NS>{});
        const uint8_t *const as = lds[BUF];
        const uint8_t *const bs = as + A_STAGE;
        auto across = [&](const uint8_t *p, int pitch) __attribute__((always_inline)) {
            const u32x2_t lo = lds_read_tr<DT_BF16>(p), hi = lds_read_tr<DT_BF16>(p + 4 * pitch);
            return u32x4_t{lo[0], lo[1], hi[0], hi[1]};
        };
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            u32x4_t fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                // rows 32 further down: the chunk of k-step st ^ 2
                if constexpr (L::AT) fa[i] = across(as + at_fo[i] + 16 * st * A_PITCH, A_PITCH);
                else fa[i] = *reinterpret_cast<const u32x4_t *>(as + a_fo[st ^ (2 * (i & 1))] + 4096 * i);
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                if constexpr (L::BT) {
                    // HALF rows further down: 32 rows an odd or even number of times
                    fb[j] = *reinterpret_cast<const u32x4_t *>(bs + bt_fo[st ^ (2 * (j * (HALF / 32) & 1))] + HALF * 128 * j);
                } else {
                    fb[j] = across(bs + b_fo[j] + 16 * st * B_PITCH, B_PITCH);
                }
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = mfma32<DT_BF16>(fa[i], fb[j], acc[i][j]);
        }
    };

    if (nk > 0) {
        static_for<0, NS - 1>([&](auto u) { load_stage(decltype(u)::value, u); });
        if constexpr (L::EXPAND)
            if (work.slice == 0) expand_adapters<OP == FUSED_ADAPT, HALF>(a, acc, m0 + wrow0, n0 + wcol0, lane);
        for (int kt = 0; kt < nk; kt += NS) {
            static_for<0, NS>([&](auto u) {
                if (kt + decltype(u)::value < nk) iteration(kt + decltype(u)::value, u);
            });
        }
    } else if constexpr (L::EXPAND) {
        if (work.slice == 0) expand_adapters<OP == FUSED_ADAPT, HALF>(a, acc, m0 + wrow0, n0 + wcol0, lane);
    }
    stage_barrier();       // drains the loads past the end before sum_slices borrows a word of the buffers
    if (work.slices > 1 &&
        !sum_slices<THREADS>(a.g, acc, work.slot, work.slice, work.slices, M - (m0 + wrow0), *reinterpret_cast<int *>(lds[0])))
        return;
    store_fused<OP, THREADS, HALF>(a, acc, which, m0 + wrow0, n0 + wcol0, lane);
}

}  // namespace gemm
