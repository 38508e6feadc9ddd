// kern_fused_pingpong.h -- the fused products on output tiles of 128 to 256 x 256, two wave groups in turn.
#pragma once

#include "kern_fused_tile.h"

namespace gemm {

// ---------------------------------------------------------------------------
// gemm_pingpong_kernel's plan for the fused products: 8 waves in two groups that alternate between reading
// fragments and running MFMAs, two LDS stages of 64 k of four units each, every unit refilled as soon as both groups have read it
// (that kernel's comment gives the order of all accesses).  BM = 64 (H0 + H1): a wave owns H0 + H1 fragment
// rows, H0 of them in unit A0 and H1 in A1, so 256, 192 and 128 rows share the code and a tile can be chosen whose
// count fills whole rounds of the 256 compute units.  The units B0 and B1 are the tile's column halves; GATED
// takes them from the two weights, so that a lane ends with g and u of the same outputs and the activation costs
// no exchange.
//
// A phase waits until its successor's unit has landed: all but the loads of the last six units, of which three are
// B's, and of A0 and A1 two and one or one and two.
//
// Bound by the MFMAs at the clock that the power limit leaves with 256 rows (a stage of 64 k takes 1.6 us: 1330 TFLOP/s on a
// full chip), by the load path with 128 (48 KB in 0.95 us).  Measured: gated 2048 x 11008 x 4096 with G and U kept 302 to
// 316 us (tile kernel: 541), dx 2048 x 4096 x 2 . 11008 in two slices 283 to 294 (529), both weight gradients
// 11008 x 4096 x 2048 304 to 329 (507).
// ---------------------------------------------------------------------------
template <int OP, int H0, int H1>
__device__ __forceinline__ void fused_pingpong_tile(const FusedArgs &a, const FusedWork &work, uint8_t *buffers, int wave, int lane) {
    using L = FusedLayout<OP>;
    constexpr int BK = 64, WAVES = 8, TM = H0 + H1, TN = 2, BM = 64 * TM, BN = 256, HALF = 128;
    constexpr int A0_BYTES = 64 * H0 * 128, A1_BYTES = 64 * H1 * 128, B_BYTES = HALF * 128;
    constexpr int STAGE = A0_BYTES + A1_BYTES + 2 * B_BYTES;
    constexpr int LB = 2, WAIT_A0 = 3 * LB + 2 * H0 + H1, WAIT_A1 = 3 * LB + H0 + 2 * H1;     // loads: H0, H1 and LB a unit
    constexpr int B_PITCH = L::BT ? 128 : HALF * 2, B_CPR = B_PITCH / 16;
    constexpr int COLS = BN / L::HALVES;
    enum { U_B0, U_A0, U_B1, U_A1 };                       // units of a stage, in load order
    constexpr int AT_B0 = 0, AT_A0 = B_BYTES, AT_B1 = AT_A0 + A0_BYTES, AT_A1 = AT_B1 + B_BYTES;


    uint8_t *const lds[2] = {buffers, buffers + STAGE};
    const int grp = wave >> 2, wave_n = wave & 3;
    const int64_t M = a.g.M, N = a.g.N, m0 = work.m0, n0 = work.n0;
    const int K = int(a.g.K), one = (K + BK - 1) / BK;      // stages of one product
    const int which = work.which, first = work.first, ns = work.count;
    const uint8_t *const a_src = static_cast<const uint8_t *>(which ? a.A2 : a.g.A);
    const int lda_b = int(which ? a.lda2 : a.g.lda) * 2, lda2_b = int(a.lda2) * 2;       // at most 4 MiB
    const int ldb_b = int(a.g.ldb) * 2, ldb2_b = int(a.ldb2) * 2;
    const int rows_valid = M - m0 < BM ? int(M - m0) : BM, cols_valid = N - n0 < COLS ? int(N - n0) : COLS;

    // ---- global source offsets of this lane's pieces: load i of a unit fills its bytes [(8 i + wave) KiB, + 1 KiB) ----
    uint32_t a_voff[TM], a2_voff[TM];                      // A0's H0 loads, then A1's
    int a_chunk[TM];
    static_for<0, TM>([&](auto v_c) __attribute__((always_inline)) {
        constexpr int V = decltype(v_c)::value, H = V < H0 ? H0 : H1, I = V < H0 ? V : V - H0, BASE = V < H0 ? 0 : 32 * H0;
        // Unit row (or column, across k) u is the tile's (u / (32 H)) * 32 TM + BASE + u % (32 H).
        if constexpr (L::AT) {
            constexpr int CPR = 8 * H;
            const int k = (I * WAVES + wave) * (64 / CPR) + lane / CPR;
            const int u = 8 * ((lane % CPR) ^ ring_bswz<DT_BF16, CPR>(k));
            const int c = u / (32 * H) * (32 * TM) + BASE + u % (32 * H);
            a_chunk[V] = 0;
            a_voff[V] = m0 + c < M ? uint32_t(k * lda_b + c * 2) : kOOB;
        } else {
            const int u = (I * WAVES + wave) * 8 + (lane >> 3);
            const int row = u / (32 * H) * (32 * TM) + BASE + u % (32 * H);
            a_chunk[V] = swz(lane & 7, u);
            a_voff[V] = uint32_t(row * lda_b + a_chunk[V] * 16);
            a2_voff[V] = uint32_t(row * lda2_b + a_chunk[V] * 16);
        }
    });
    uint32_t b_voff[2][LB], b2_voff[2][LB];                // by half
    int b_chunk[LB];
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        if constexpr (L::BT) {
            const int row = (i * WAVES + wave) * 8 + (lane >> 3);
            b_chunk[i] = swz(lane & 7, row);
            b_voff[0][i] = uint32_t(row * ldb_b + b_chunk[i] * 16);
            b_voff[1][i] = L::HALVES == 2 ? uint32_t(row * ldb2_b + b_chunk[i] * 16) : uint32_t((HALF + row) * ldb_b + b_chunk[i] * 16);
        } else {
            const int k = (i * WAVES + wave) * (1024 / B_PITCH) + lane / B_CPR;
            const int c = 8 * ((lane % B_CPR) ^ ring_bswz<DT_BF16, B_CPR>(k));
            b_chunk[i] = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = n0 + h * HALF + c < N;
                b_voff[h][i] = in ? uint32_t(k * ldb_b + (h * HALF + c) * 2) : kOOB;
                b2_voff[h][i] = in ? uint32_t(k * ldb2_b + (h * HALF + c) * 2) : kOOB;
            }
        }
    }
    // Where the tile's operands begin at k = 0.
    const uint8_t *const a_base = a_src + (L::AT ? m0 * 2 : m0 * lda_b);
    const uint8_t *const a2_base = static_cast<const uint8_t *>(a.A2) + m0 * lda2_b;
    const uint8_t *const b_base = static_cast<const uint8_t *>(a.g.B) + (L::BT ? n0 * ldb_b : n0 * 2);
    const uint8_t *const b2_base = static_cast<const uint8_t *>(a.B2) + (L::BT ? n0 * ldb2_b : n0 * 2);

    // Issues this wave's loads of unit U of stage kt (buffer BUF).
    auto load_unit = [&](int kt, auto buf_c, auto u_c) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_c)::value, U = decltype(u_c)::value;
        int t = first + kt;
        const bool live = kt < ns, second = OP == FUSED_DX && t >= one;
        if (second) t -= one;
        const int rem = live ? (K - t * BK < BK ? K - t * BK : BK) : 0;
        if constexpr (U == U_A0 || U == U_A1) {
            constexpr int V0 = U == U_A0 ? 0 : H0, COUNT = U == U_A0 ? H0 : H1;
            const uint32_t dst = lds_addr(lds[BUF]) + (U == U_A0 ? AT_A0 : AT_A1) + uint32_t(wave) * 1024u;
            const int ld = second ? lda2_b : lda_b;
            const i32x4_t r = ring_rsrc((second ? a2_base : a_base) + (L::AT ? int64_t(t) * BK * ld : int64_t(t) * (2 * BK)),
                                        uint32_t(__builtin_amdgcn_readfirstlane((L::AT ? rem : rem > 0 ? rows_valid : 0) * ld)));
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
                ring_load16(r, dst + i * (WAVES * 1024),
                            L::AT || a_chunk[V0 + i] * 8 < rem ? (!L::AT && second ? a2_voff[V0 + i] : a_voff[V0 + i]) : kOOB);
        } else {
            constexpr int H = U == U_B1 ? 1 : 0;
            const uint32_t dst = lds_addr(lds[BUF]) + (H ? AT_B1 : AT_B0) + uint32_t(wave) * 1024u;
            if constexpr (L::BT) {
                const bool up = L::HALVES == 2 && H == 1;
                const i32x4_t r = ring_rsrc((up ? b2_base : b_base) + int64_t(t) * (2 * BK),
                                            uint32_t(__builtin_amdgcn_readfirstlane(rem > 0 ? cols_valid * (up ? ldb2_b : ldb_b) : 0)));
#pragma unroll
                for (int i = 0; i < LB; ++i) ring_load16(r, dst + i * (WAVES * 1024), b_chunk[i] * 8 < rem ? b_voff[H][i] : kOOB);
            } else {
                const int ld = second ? ldb2_b : ldb_b;
                const i32x4_t r = ring_rsrc((second ? b2_base : b_base) + int64_t(t) * BK * ld,
                                            uint32_t(__builtin_amdgcn_readfirstlane(rem * ld)));
#pragma unroll
                for (int i = 0; i < LB; ++i) ring_load16(r, dst + i * (WAVES * 1024), second ? b2_voff[H][i] : b_voff[H][i]);
            }
        }
    };

    // ---- fragment offsets within a unit ----
    const int frag_row = lane & 31, frag_half = lane >> 5;
    int a_fo[2][4], bt_fo[4];                              // along k: k-step st of the wave's first 32 rows of A0, A1
#pragma unroll
    for (int st = 0; st < 4; ++st) {
        const int ra0 = grp * 32 * H0 + frag_row, ra1 = grp * 32 * H1 + frag_row, rb = wave_n * 32 + frag_row;
        a_fo[0][st] = ra0 * 128 + 16 * swz(2 * st + frag_half, ra0);
        a_fo[1][st] = ra1 * 128 + 16 * swz(2 * st + frag_half, ra1);
        bt_fo[st] = rb * 128 + 16 * swz(2 * st + frag_half, rb);
    }
    const int lgrp = lane >> 4, g16 = lane & 15;           // across k: transpose reads, as in gemm_lds_kernel
    const int tr_row = g16 >> 2, tr_colb = (g16 & 3) * 8 + (lgrp & 1) * 32, tr_k = (lgrp >> 1) * 8 + tr_row;
    auto across_fo = [&](auto cpr_c, int col) __attribute__((always_inline)) {
        constexpr int CPR = decltype(cpr_c)::value;
        const int colb = col * 2 + tr_colb;
        return tr_k * (CPR * 16) + (((colb >> 4) ^ ring_bswz<DT_BF16, CPR>(tr_row)) << 4) + (colb & 15);
    };
    int at_fo[TM];
    static_for<0, TM>([&](auto v_c) __attribute__((always_inline)) {
        constexpr int V = decltype(v_c)::value, H = V < H0 ? H0 : H1, I = V < H0 ? V : V - H0;
        at_fo[V] = across_fo(std::integral_constant<int, 8 * H>{}, grp * 32 * H + 32 * I);
    });
    const int b_fo = across_fo(std::integral_constant<int, HALF / 8>{}, wave_n * 32);

    constexpr int HM = H0 > H1 ? H0 : H1;
    u32x4_t fa[HM][4], fb[2][4];                           // A: one unit's fragment rows; B: halves 0 and 1; four k-steps
    auto across = [&](const uint8_t *p, int pitch) __attribute__((always_inline)) {
        const u32x2_t lo = lds_read_tr<DT_BF16>(p), hi = lds_read_tr<DT_BF16>(p + 4 * pitch);
        return u32x4_t{lo[0], lo[1], hi[0], hi[1]};
    };
    auto read_a = [&](auto buf_c, auto u_c) __attribute__((always_inline)) {
        constexpr int H = decltype(u_c)::value == U_A1, N_ROWS = H ? H1 : H0;
        const uint8_t *const p = lds[decltype(buf_c)::value] + (H ? AT_A1 : AT_A0);
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < N_ROWS; ++i) {
                if constexpr (L::AT) {
                    fa[i][st] = across(p + at_fo[(H ? H0 : 0) + i] + 16 * st * (128 * N_ROWS), 128 * N_ROWS);
                } else {
                    // the swizzle of rows 32 further down differs by chunk ^ 4: k-step st ^ 2's chunk
                    fa[i][st] = *reinterpret_cast<const u32x4_t *>(p + a_fo[H][st ^ (2 * (i & 1))] + 4096 * i);
                }
            }
    };
    auto read_b = [&](auto buf_c, auto u_c) __attribute__((always_inline)) {
        constexpr int H = decltype(u_c)::value == U_B1;
        const uint8_t *const p = lds[decltype(buf_c)::value] + (H ? AT_B1 : AT_B0);
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            if constexpr (L::BT) fb[H][st] = *reinterpret_cast<const u32x4_t *>(p + bt_fo[st]);
            else fb[H][st] = across(p + b_fo + 16 * st * B_PITCH, B_PITCH);
        }
    };

    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};

    // Ends a phase's reads and loads, then runs its quadrant (unit A_H, column half J).
    auto quadrant = [&](auto h_c, auto j_c, auto wait_c) __attribute__((always_inline)) {
        constexpr int H = decltype(h_c)::value, J = decltype(j_c)::value, V0 = H ? H0 : 0, COUNT = H ? H1 : H0;
        __builtin_amdgcn_sched_barrier(0);
        ring_barrier<decltype(wait_c)::value>();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) acc[V0 + i][J] = mfma32<DT_BF16>(fa[i][st], fb[J][st], acc[V0 + i][J]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using B0 = std::integral_constant<int, U_B0>;
    using A0 = std::integral_constant<int, U_A0>;
    using B1 = std::integral_constant<int, U_B1>;
    using A1 = std::integral_constant<int, U_A1>;
    // The last six units after a load of B0 or A1 hold two A1's, after one of A0 or B1 two A0's.
    using W0 = std::integral_constant<int, WAIT_A0>;
    using W1 = std::integral_constant<int, WAIT_A1>;
    auto stage = [&](int kt, auto buf_c) __attribute__((always_inline)) {
        using NEXT = std::integral_constant<int, 1 - decltype(buf_c)::value>;
        read_a(buf_c, A0{});
        load_unit(kt + 2, buf_c, B0{});
        quadrant(I0{}, I0{}, W1{});
        read_b(buf_c, B1{});
        load_unit(kt + 2, buf_c, A0{});
        quadrant(I0{}, I1{}, W0{});
        read_a(buf_c, A1{});
        load_unit(kt + 2, buf_c, B1{});
        quadrant(I1{}, I0{}, W0{});
        read_b(NEXT{}, B0{});
        load_unit(kt + 2, buf_c, A1{});
        quadrant(I1{}, I1{}, W1{});
    };

    if (ns > 0) {
        static_for<0, 2>([&](auto s) {
            load_unit(decltype(s)::value, s, B0{});
            load_unit(decltype(s)::value, s, A0{});
            load_unit(decltype(s)::value, s, B1{});
            load_unit(decltype(s)::value, s, A1{});
        });
    }
    if constexpr (L::EXPAND)
        if (work.slice == 0) expand_adapters<OP == FUSED_ADAPT, HALF>(a, acc, m0 + grp * (32 * TM), n0 + wave_n * 32, lane);
    if (ns > 0) {
        // B0 and A0 of stage 0 have landed: all but the other six units.
        ring_barrier<3 * LB + H0 + 2 * H1>();
        read_b(I0{}, B0{});
        phase_barrier();                                   // ... and B0 is read, before phase 1 refills it
        if (grp == 1) asm volatile("s_barrier" ::: "memory");
        int kt = 0;
        for (; kt + 1 < ns; kt += 2) {
            stage(kt, I0{});
            stage(kt + 1, I1{});
        }
        if (kt < ns) stage(kt, I0{});
        if (grp == 0) asm volatile("s_barrier" ::: "memory");
    }
    stage_barrier();                                       // drains the loads past the end, by every wave
    if (work.slices > 1 &&
        !sum_slices<512>(a.g, acc, work.slot, work.slice, work.slices, M - (m0 + grp * (32 * TM)), *reinterpret_cast<int *>(lds[0])))
        return;
    store_fused<OP, 512, HALF>(a, acc, which, m0 + grp * (32 * TM), n0 + wave_n * 32, lane);
}

// Tiles of 64 (H0 + H1) rows, and where L0 > 0 lower ones of 64 (L0 + L1) rows in a last round.
template <int OP, int H0, int H1, int L0, int L1>
__global__ __attribute__((amdgpu_flat_work_group_size(512, 512), amdgpu_waves_per_eu(2, 2)))
void fused_pingpong_kernel(FusedArgs a) {
    __shared__ __attribute__((aligned(1024))) uint8_t buffers[2 * (64 * (H0 + H1) + 256) * 128];
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), lane = int(threadIdx.x) & 63;
    const int one = (int(a.g.K) + 63) / 64;
    const FusedWork work = fused_work<64 * (H0 + H1), 64 * (L0 + L1), 256 / FusedLayout<OP>::HALVES>(a, OP == FUSED_DX ? 2 * one : one);
    if constexpr (L0 > 0) {
        if (work.low) {
            fused_pingpong_tile<OP, L0, L1>(a, work, buffers, wave, lane);
            return;
        }
    }
    fused_pingpong_tile<OP, H0, H1>(a, work, buffers, wave, lane);
}

}  // namespace gemm
