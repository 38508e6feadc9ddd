// kern_mx_tile.h -- the products over block-scaled operands on output tiles.
#pragma once

#include "mx_common.h"

namespace gemm {

// Adds the sums of WK groups of waves up, in their order, into the first group's registers,
// through `bytes` of LDS that nothing else uses any more, in as many passes as that takes.
template <int WK, int BYTES, int TM, int TN>
__device__ __forceinline__ void mx_sum_groups(f32x16_t (&acc)[TM][TN], uint8_t *lds, int group, int tid) {
    if constexpr (WK > 1) {
        f32x4_t *const sums = reinterpret_cast<f32x4_t *>(lds);
        const int own = int(blockDim.x) / WK;
        constexpr int SLOTS = TM * TN * 4, MOST = BYTES / 16;      // values that fit; own <= 512
        auto pass = [&](auto first_c, auto count_c) __attribute__((always_inline)) {
            constexpr int FIRST = decltype(first_c)::value, COUNT = decltype(count_c)::value;
            if (group > 0) {
#pragma unroll
                for (int v = FIRST; v < FIRST + COUNT; ++v) {
                    const f32x16_t &x = acc[v / 4 / TN][v / 4 % TN];
                    const int q = 4 * (v % 4);
                    sums[((group - 1) * COUNT + v - FIRST) * own + tid - group * own] = f32x4_t{x[q], x[q + 1], x[q + 2], x[q + 3]};
                }
            }
            phase_barrier();
            if (group == 0) {
#pragma unroll
                for (int o = 0; o < WK - 1; ++o)
#pragma unroll
                    for (int v = FIRST; v < FIRST + COUNT; ++v) {
                        const f32x4_t x = sums[(o * COUNT + v - FIRST) * own + tid];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[v / 4 / TN][v / 4 % TN][4 * (v % 4) + e] += x[e];
                    }
            }
            phase_barrier();
        };
        constexpr int OWN = 256;                                    // most threads of a group that take several passes
        constexpr int FIT = MOST / ((WK - 1) * OWN) < 1 ? 1 : MOST / ((WK - 1) * OWN);
        constexpr int COUNT = SLOTS <= FIT ? SLOTS : FIT >= SLOTS / 2 ? SLOTS / 2 : SLOTS / 4;
        static_assert((WK - 1) * COUNT * OWN * 16 <= BYTES, "a pass fits");
        static_for<0, SLOTS / COUNT>([&](auto p) {
            pass(std::integral_constant<int, decltype(p)::value * COUNT>{}, std::integral_constant<int, COUNT>{});
        });
    }
}

// ---------------------------------------------------------------------------
// C = A . W^T, W 4-bit N x K.  Both operands go from memory straight into a ring of NS LDS
// stages of KS k: A as BM rows of 128 bytes per 64 k (16-byte chunks XOR-swizzled by swz), W
// packed as it is, BN rows of KS / 2 bytes.  A lane reads the 16 bytes of one W block once
// (32 k: its share of four MFMA k-steps) and converts eight codes at a time in registers,
// so W costs a quarter of bf16's LDS and load-path traffic and the conversions (four
// instructions per 32 x 16 fragment) are repeated only by the WM waves that share its rows.
// k-step t of a 64-k part takes, for lanes of half h, k = 32 h + 8 t + 0..7 of both operands.
//
// The block scales of the tile's rows sit in LDS for PANEL k at a time, loaded ahead of the
// first stage and again between two stages: their bytes are too few and too scattered to
// ride along in each stage.  Straight into LDS where their rows are on dwords; through
// registers elsewhere, which waits for the stages on their way too.
//
// WK > 1: that many groups of waves take turns at the 64-k parts of a stage, and add their
// sums up in LDS at the end.  A narrow tile's wave has one or two fragments, and its k-steps wait
// for each other (LDS read, conversion, MFMA: 1000 clocks per 128 k with one wave per
// SIMD); a second wave fills those waits without more K slices to sum.
//
// Measured: 2048 x 11008 x 4096 154 to 164 us (1130 to 1200 TFLOP/s; the matrix unit busy 51 % of the
// clocks, the compute units 85 %: 1.85 rounds of 192 x 256 tiles; waves waiting 37 % of theirs); 16 x 4096 x 14336 12.7 us, of which the K loop
// ends at 7.5 (46 GB/s per CU, what the load path gives) and the slices' sum takes 4.5.
// Against it, at 2048 x 11008 x 4096: 128 x 256 tiles at four waves per SIMD 165 to 180 us (spills), stages
// of 64 k 158 (128 x 256) and 164; a stage's loads all at once a few per cent more.
// ---------------------------------------------------------------------------
template <int BM, int BN, int WM, int WN, int WK, int WAVES_PER_EU, int KS, int NS, int PANEL>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * WM * WN * WK, 64 * WM * WN * WK),
                          amdgpu_waves_per_eu(WAVES_PER_EU, WAVES_PER_EU)))
void mx_fwd_kernel(MxArgs a) {
    constexpr int WAVES = WM * WN * WK, THREADS = 64 * WAVES;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int PARTS = KS / 64;                            // 64-k parts of a stage
    constexpr int A_PART = BM * 128, A_STAGE = A_PART * PARTS;
    constexpr int PITCH = KS / 2, CPR = PITCH / 16;           // bytes and chunks of a W row
    constexpr int B_STAGE = BN * PITCH;
    constexpr int A_INSTR = A_STAGE / 1024 / WAVES, B_INSTR = B_STAGE / 1024 / WAVES;
    constexpr int LPS = A_INSTR + B_INSTR;
    static_assert(A_INSTR >= 1 && A_INSTR * 1024 * WAVES == A_STAGE, "A stage split");
    static_assert(B_INSTR >= 1 && B_INSTR * 1024 * WAVES == B_STAGE, "W stage split");
    static_assert(NS >= 2 && (NS - 1) * LPS < 64, "loads in flight must fit vmcnt");
    // A panel row is P_CPR chunks of 16 scales; chunk c of row r sits at chunk c ^ p_swz(r), which
    // puts 16 consecutive rows' scales of one block on different banks.
    constexpr int P_PITCH = PANEL / kMxBlock, P_CPR = P_PITCH / 16;
    static_assert(PANEL % KS == 0 && P_CPR >= 1 && P_CPR <= 8 && (P_CPR & (P_CPR - 1)) == 0, "panel rows");
    constexpr int P_BYTES = (BN * P_PITCH + 1024 * WAVES - 1) / (1024 * WAVES) * (1024 * WAVES);
    constexpr int P_INSTR = P_BYTES / (256 * WAVES);           // dword loads per lane
    static_assert((NS - 1) * LPS + P_INSTR < 64, "loads in flight must fit vmcnt");
    static_assert(PARTS % WK == 0, "the groups have as many parts of a stage each");
    static_assert(WK == 1 || THREADS / WK <= 256, "mx_sum_groups");

    __shared__ __attribute__((aligned(1024))) uint8_t lds[NS][A_STAGE + B_STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t panel[P_BYTES];

    const int tid = int(threadIdx.x), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = wave / (WM * WN), wave_m = wave / WN % WM, wave_n = wave % WN;
    int tm, tn, slice;
    map_tile(a.g, tm, tn, slice);
    const int64_t M = a.g.M, N = a.g.N;
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
    const int64_t k_begin = int64_t(slice) * a.g.k_chunk;
    const int64_t k_end = k_begin + a.g.k_chunk < a.g.K ? k_begin + a.g.k_chunk : a.g.K;
    const int k_len = k_end > k_begin ? int(k_end - k_begin) : 0;
    const int nk = (k_len + KS - 1) / KS;
    const int64_t lda_b = a.g.lda * 2, ldq = a.g.ldb;

    // Where this lane's pieces of a stage come from.  A: load i fills part (i W + wave) KiB / A_PART.
    const uint32_t a_bytes = uint32_t(((M - m0) < BM ? (M - m0) : BM) * lda_b);
    uint32_t a_voff[A_INSTR];
    int a_k[A_INSTR];
#pragma unroll
    for (int i = 0; i < A_INSTR; ++i) {
        const int row = ((i * WAVES + wave) * 8 + (lane >> 3)) % BM, part = ((i * WAVES + wave) * 8) / BM;
        const int c = swz(lane & 7, row);
        a_k[i] = 64 * part + 8 * c;
        a_voff[i] = uint32_t(row * lda_b + 128 * part + 16 * c);
    }
    // W: chunk c of row r sits at chunk c ^ w_swz(r), which spreads 32 rows' reads over the banks.
    auto w_swz = [](int row) { return CPR == 8 ? (row ^ (row >> 3)) & 7 : CPR == 4 ? ring_swz(row) : (row >> 3) & 1; };
    const uint32_t b_bytes = uint32_t(((N - n0) < BN ? (N - n0) : BN) * ldq);
    uint32_t b_voff[B_INSTR];
    int b_k[B_INSTR];
#pragma unroll
    for (int i = 0; i < B_INSTR; ++i) {
        const int row = (i * WAVES + wave) * (64 / CPR) + lane / CPR;
        const int c = (lane % CPR) ^ w_swz(row);
        b_k[i] = 32 * c;
        b_voff[i] = uint32_t(row * ldq + 16 * c);
    }
    const uint8_t *const a_base = static_cast<const uint8_t *>(a.g.A) + m0 * lda_b + k_begin * 2;
    const uint8_t *const b_base = static_cast<const uint8_t *>(a.g.B) + n0 * ldq + k_begin / 2;

    // Loads FROM .. TO - 1 of a stage's LPS (W's first).  A stage's loads go out a few with each
    // k-step: all at once they back up the vector memory path, and every wave of the
    // workgroup waits behind them at the same time instead of multiplying.
    auto load_some = [&](int kt, auto buf_c, auto from_c, auto to_c) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_c)::value, FROM = decltype(from_c)::value, TO = decltype(to_c)::value;
        const int rem = k_len - kt * KS;
        const uint32_t dst = lds_addr(lds[BUF]) + uint32_t(wave) * 1024u;
        const i32x4_t ra = ring_rsrc(uniform(a_base + int64_t(kt) * (KS * 2)), uniform(rem > 0 ? a_bytes : 0u));
        const i32x4_t rb = ring_rsrc(uniform(b_base + int64_t(kt) * PITCH), uniform(rem > 0 ? b_bytes : 0u));
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            if (i < B_INSTR) {
                ring_load16(rb, dst + A_STAGE + i * (WAVES * 1024), b_k[i] < rem ? b_voff[i] : kOOB);
            } else {
                const int j = i - B_INSTR;
                ring_load16(ra, dst + j * (WAVES * 1024), a_k[j] < rem ? a_voff[j] : kOOB);
            }
        }
    };
    auto load_stage = [&](int kt, auto buf_c) __attribute__((always_inline)) {
        load_some(kt, buf_c, std::integral_constant<int, 0>{}, std::integral_constant<int, LPS>{});
    };
    // The scales of rows n0.. from k0 (of this slice) on, 16 or 4 bytes at a time where rows and
    // addresses allow it, else byte by byte.  Rows past N take 0; a row's last piece may go on
    // past its last block, within its stride or (in the matrix' last row) an aligned piece
    // that holds one: those scales are made 0 where they are read (`blocks` below).
    auto p_swz = [](int row) { return (row / (16 / P_CPR)) & (P_CPR - 1); };
    const uint64_t scale_bits = reinterpret_cast<uintptr_t>(a.scales) | uint64_t(a.ld_scales) |
                                (a.ld_scales < (int64_t(1) << 22) ? 0u : 1u);
    auto load_panel = [&](int k0) __attribute__((always_inline)) {
        const int64_t b0 = (k_begin + k0) / kMxBlock, nb = (a.g.K + kMxBlock - 1) / kMxBlock;
        const int64_t rows = N - n0 < BN ? N - n0 : BN;
        if ((scale_bits & 3) != 0) {
            for (int p = tid; p < BN * P_PITCH / 4; p += THREADS) {
                const int r = p / (P_PITCH / 4), d = p % (P_PITCH / 4);
                const uint8_t *const src = a.scales + (n0 + r) * a.ld_scales + b0 + 4 * d;
                const int64_t left = r < rows ? nb - (b0 + 4 * d) : 0;
                uint32_t v = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < left) v |= uint32_t(src[e]) << (8 * e);
                *reinterpret_cast<uint32_t *>(&panel[r * P_PITCH + 16 * ((d / 4) ^ p_swz(r)) + 4 * (d % 4)]) = v;
            }
            return;
        }
        const i32x4_t rs = ring_rsrc(uniform(a.scales + n0 * a.ld_scales + b0), 0x7fffffffu);
        if ((scale_bits & 15) == 0 && b0 % 16 == 0) {
#pragma unroll
            for (int i = 0; i < P_INSTR / 4; ++i) {
                const int p = (i * WAVES + wave) * 64 + lane, r = p / P_CPR, c = (p % P_CPR) ^ p_swz(r);
                const bool in = r < rows && b0 + 16 * c < nb;
                ring_load16(rs, lds_addr(panel) + uint32_t(i * WAVES + wave) * 1024u, in ? uint32_t(r * a.ld_scales + 16 * c) : kOOB);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < P_INSTR; ++i) {
                const int p = (i * WAVES + wave) * 64 + lane, r = p / (P_PITCH / 4), d = p % (P_PITCH / 4);
                const int c = (d / 4) ^ p_swz(r);
                const bool in = r < rows && b0 + 16 * c + 4 * (d % 4) < nb;
                ring_load4(rs, lds_addr(panel) + uint32_t(i * WAVES + wave) * 256u,
                           in ? uint32_t(r * a.ld_scales + 16 * c + 4 * (d % 4)) : kOOB);
            }
        }
    };
    const int blocks = (k_len + kMxBlock - 1) / kMxBlock;      // of this slice

    const int frag_row = lane & 31, half = lane >> 5;
    const int r0 = wave_m * (BM / WM) + frag_row, c0 = wave_n * (BN / WN) + frag_row;
    int a_fo[2][4];                                           // k-step t of the wave's 32-row tiles (even, odd)
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int t = 0; t < 4; ++t) a_fo[p][t] = r0 * 128 + 16 * (swz(4 * half + t, r0) ^ (4 * p));
    int b_fo[TN][PARTS / WK];                                  // this group's parts
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int p = 0; p < PARTS / WK; ++p)
            b_fo[j][p] = A_STAGE + (c0 + 32 * j) * PITCH + 16 * ((2 * (p * WK + group) + half) ^ w_swz(c0 + 32 * j));

    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};

    // Fragments of two k-steps: one multiplied while the next is read and converted.
    u32x4_t fa[2][TM], fb[2][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[1][i] = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[1][j] = u32x4_t{0u, 0u, 0u, 0u};
    auto multiply = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mfma32<DT_BF16>(fa[slot][i], fb[slot][j], acc[i][j]);
    };
    // One stage.  Slot 1 holds the fragments of the k-step before, whose MFMAs run under the
    // latency of this stage's first reads.
    auto iteration = [&](int kt, auto buf_c) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_c)::value;
        ring_barrier<(NS - 2) * LPS>();
        uint8_t *const st = lds[BUF];
        if (kt == nk - 1 && (k_len & 31) != 0) {
            // K ends inside a block: the codes that follow it may stand for infinities, which A's zeros
            // would make NaN.  Inside a chunk: what follows it in A's row is not part of the sum.
            const int kl = k_len - kt * KS, part = kl / 64, c = (kl % 64) / 8;
            for (int r = tid; r < BN; r += THREADS) {
                u32x4_t *const w = reinterpret_cast<u32x4_t *>(st + A_STAGE + r * PITCH + 16 * ((kl / 32) ^ w_swz(r)));
                *w = mx4_first(*w, kl % 32);
            }
            if ((kl & 7) != 0)
                for (int r = tid; r < BM; r += THREADS)
                    for (int e = kl & 7; e < 8; ++e)
                        reinterpret_cast<uint16_t *>(st + part * A_PART + r * 128 + 16 * swz(c, r))[e] = 0;
            phase_barrier();
        }
        const int block0 = (kt * KS % PANEL) / kMxBlock + half;
        static_for<0, PARTS / WK>([&](auto p_c) __attribute__((always_inline)) {
            constexpr int p = decltype(p_c)::value;
            const int q = p * WK + group, b = block0 + 2 * q;
            const bool in = kt * (KS / kMxBlock) + half + 2 * q < blocks;     // past the end: no NaN for A's zeros
            u32x4_t w[TN];
            float s[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int r = c0 + 32 * j;
                w[j] = *reinterpret_cast<const u32x4_t *>(st + b_fo[j][p]);
                s[j] = mx4_scale(in ? panel[r * P_PITCH + 16 * ((b >> 4) ^ p_swz(r)) + (b & 15)] : 0);
            }
            static_for<0, 4>([&](auto t_c) __attribute__((always_inline)) {
                constexpr int t = decltype(t_c)::value, STEP = 4 * p + t, STEPS = 4 * PARTS / WK;
                load_some(kt + NS - 1, std::integral_constant<int, (BUF + NS - 1) % NS>{},
                          std::integral_constant<int, STEP * LPS / STEPS>{}, std::integral_constant<int, (STEP + 1) * LPS / STEPS>{});
#pragma unroll
                for (int i = 0; i < TM; ++i)
                    fa[t & 1][i] = *reinterpret_cast<const u32x4_t *>(st + q * A_PART + a_fo[i & 1][t] + 4096 * i);
                multiply(1 - (t & 1));
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[t & 1][j] = mx4_to_bf16(w[j][t], s[j]);
                __builtin_amdgcn_sched_barrier(0);        // one k-step ahead, no further: registers
            });
        });
    };

    if (nk > 0) {
        load_panel(0);
        static_for<0, NS - 1>([&](auto u) { load_stage(decltype(u)::value, u); });
        for (int kt = 0; kt < nk; kt += NS) {
            static_for<0, NS>([&](auto u) {
                constexpr int U = decltype(u)::value;
                if (kt + U < nk) {
                    if (kt + U > 0 && (kt + U) % (PANEL / KS) == 0) {
                        phase_barrier();                      // every wave is done with the panel before
                        load_panel((kt + U) * KS);
                        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    }
                    iteration(kt + U, u);
                }
            });
        }
        multiply(1);
    }
    stage_barrier();
    mx_sum_groups<WK, NS * (A_STAGE + B_STAGE)>(acc, &lds[0][0], group, tid);
    mx_store_tile<BM, BN, TM, TN>(a.g, acc, tm, tn, slice, m0 + wave_m * (BM / WM), n0 + wave_n * (BN / WN), lane,
                                  group == 0, *reinterpret_cast<int *>(lds[0]));
}

// ---------------------------------------------------------------------------
// C = A . W (MX_DX: A bf16 M x K, W 4-bit K x N) and C = A^T . X (MX_DW: A bf16 K x M, X 8-bit
// K x N): the blocks lie along N, across the sum, so every k of a column has another scale
// and no scale can be applied after the matrix instruction.  B is converted to bf16 (exactly)
// once per workgroup, on its way into LDS: a thread takes one block of 32 codes of one row k
// through registers per stage.  A goes straight from memory into LDS.  A stage is 64 k for
// each of WK groups of waves, which add their sums up at the end (as mx_fwd_kernel's).
//
// LDS, two stages each: A as BM rows of 128 bytes per 64 k (DX), or as rows (k) of BM elements read
// back transposed (DW), both as gemm_lds_kernel lays them out.  B in one region per block column:
// rows (k) of 32 bf16, the 64-byte rows back to back, the regions 64 bytes further apart.
// A transpose read then covers two runs of 256 bytes, and the eight lanes that write one row's
// chunks hit different banks (the regions of blocks 0-3 by their offset, 4-7 by a flipped chunk).
//
// B's codes are loaded two stages ahead into registers, A one stage ahead into LDS.
//
// Few rows are mx_rows_kernel's.
//
// Measured: DX 2048 x 4096 x 11008 158 to 167 us (1110 to 1170 TFLOP/s; the matrix unit busy 48 % of the
// clocks, LDS 48 %, a quarter of it bank conflicts; waves wait for LDS 20 % of their time); DW 11008 x
// 4096 x 2048 178 to 185 us (1000 to 1040 TFLOP/s; matrix unit 46 %, LDS 29 %, compute units 83 %: 2.69
// rounds of tiles, 6.4 us of stores of C in each).  Against it: A in a ring of three stages made no difference (64.3 and 64.8 us at
// 2048 x 4096 x 4096); the loads in two halves 114 against 106 us (DX 2048 x 8192 x 4096); X unpacked to
// bf16 by a launch of its own 180 against 183.5 us (DW 11008 x 4096 x 2048) but 74 against 69 (4096 x
// 4096 x 2048).
// ---------------------------------------------------------------------------
template <int OP, int BM, int BN, int WM, int WN, int WK, int WAVES_PER_EU>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * WM * WN * WK, 64 * WM * WN * WK),
                          amdgpu_waves_per_eu(WAVES_PER_EU, WAVES_PER_EU)))
void mx_grad_kernel(MxArgs a) {
    constexpr bool DW = OP == MX_DW;
    constexpr int WAVES = WM * WN * WK, THREADS = 64 * WAVES;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int BK = 64 * WK;
    constexpr int A_PART = BM * 128, A_STAGE = A_PART * WK;
    constexpr int A_PITCH = DW ? BM * 2 : 128, A_CPR = A_PITCH / 16;
    constexpr int A_INSTR = A_STAGE / 1024 / WAVES;
    constexpr int BLOCKS = BN / kMxBlock, REGION = BK * 64 + 64;
    constexpr int CODES = DW ? 32 : 16;                      // bytes of a block's codes
    constexpr int RAW = CODES / 16 + 1;                      // loads per thread and stage: codes and a scale
    static_assert(A_INSTR >= 1 && A_INSTR * 1024 * WAVES == A_STAGE, "A stage split");
    static_assert(BK * BLOCKS == THREADS, "one block of one row per thread");
    static_assert(WK == 1 || THREADS / WK <= 256, "mx_sum_groups");

    __shared__ __attribute__((aligned(1024))) uint8_t a_lds[2][A_STAGE];
    __shared__ __attribute__((aligned(1024))) uint8_t b_lds0[BLOCKS * REGION];
    __shared__ __attribute__((aligned(1024))) uint8_t b_lds1[BLOCKS * REGION];

    const int tid = int(threadIdx.x), lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = wave / (WM * WN), wave_m = wave / WN % WM, wave_n = wave % WN;
    int tm, tn, slice;
    map_tile(a.g, tm, tn, slice);
    const int64_t M = a.g.M, N = a.g.N;
    const int64_t m0 = int64_t(tm) * BM, n0 = int64_t(tn) * BN;
    const int64_t k_begin = int64_t(slice) * a.g.k_chunk;
    const int64_t k_end = k_begin + a.g.k_chunk < a.g.K ? k_begin + a.g.k_chunk : a.g.K;
    const int k_len = k_end > k_begin ? int(k_end - k_begin) : 0;
    const int nk = (k_len + BK - 1) / BK;
    const int64_t lda_b = a.g.lda * 2, ldq = a.g.ldb, lds_ = a.ld_scales;

    // ---- A: this lane's pieces of a stage.
    const uint32_t a_bytes = uint32_t(((M - m0) < BM ? (M - m0) : BM) * lda_b);     // DX: rows past M read zeros
    uint32_t a_voff[A_INSTR];
    int a_k[A_INSTR];
#pragma unroll
    for (int i = 0; i < A_INSTR; ++i) {
        if constexpr (DW) {
            const int row = (i * WAVES + wave) * (64 / A_CPR) + lane / A_CPR;
            const int c = (lane % A_CPR) ^ ring_bswz<DT_BF16, A_CPR>(row);
            a_k[i] = row;
            a_voff[i] = m0 + 8 * c < M ? uint32_t(row * lda_b + 16 * c) : kOOB;
        } else {
            const int row = ((i * WAVES + wave) * 8 + (lane >> 3)) % BM, part = ((i * WAVES + wave) * 8) / BM;
            const int c = swz(lane & 7, row);
            a_k[i] = 64 * part + 8 * c;
            a_voff[i] = uint32_t(row * lda_b + 128 * part + 16 * c);
        }
    }
    const uint8_t *const a_base = static_cast<const uint8_t *>(a.g.A) + (DW ? k_begin * lda_b + m0 * 2 : m0 * lda_b + k_begin * 2);
    // Where a wave's loads are all of one group of eight rows and that lies past M, they are left out;
    // the rows' results are not stored, whatever LDS holds.
    const bool no_a = !DW && WAVES % (BM / 8) == 0 && uniform(uint32_t(m0 + wave % (BM / 8) * 8 >= M)) != 0;
    auto load_a = [&](int kt, int buf) __attribute__((always_inline)) {
        const int rem = k_len - kt * BK;
        const uint32_t dst = lds_addr(a_lds[0]) + uint32_t(buf * A_STAGE) + uint32_t(wave) * 1024u;
        const i32x4_t ra = DW ? ring_rsrc(uniform(a_base + int64_t(kt) * BK * lda_b),
                                          uniform(uint32_t((rem <= 0 ? 0 : rem < BK ? rem : BK) * lda_b)))
                              : ring_rsrc(uniform(a_base + int64_t(kt) * (BK * 2)), uniform(rem > 0 ? a_bytes : 0u));
#pragma unroll
        for (int i = 0; i < A_INSTR; ++i)
            if (!no_a) ring_load16(ra, dst + i * (WAVES * 1024), a_k[i] < rem ? a_voff[i] : kOOB);
    };

    // ---- B: this thread's block of row b_row of each stage.
    const int b_row = tid / BLOCKS, b_blk = tid % BLOCKS;
    const bool b_in = n0 + b_blk * kMxBlock < N;
    const uint32_t q_off = uint32_t(b_row * ldq + b_blk * CODES), s_off = uint32_t(b_row * lds_ + b_blk);
    const uint8_t *const q_base = static_cast<const uint8_t *>(a.g.B) + k_begin * ldq + (DW ? n0 : n0 / 2);
    const uint8_t *const s_base = a.scales + k_begin * lds_ + n0 / kMxBlock;
    // The second half of a block's 8-bit codes may lie past N.
    const bool b_in2 = n0 + b_blk * kMxBlock + 16 < N;
    u32x4_t raw[2][CODES / 16];
    uint32_t raw_scale[2];
    auto load_b = [&](int kt, auto set_c) __attribute__((always_inline)) {
        constexpr int SET = decltype(set_c)::value;
        const bool in = b_in && kt * BK + b_row < k_len;
        const __amdgpu_buffer_rsrc_t rq = make_rsrc(q_base + int64_t(kt) * BK * ldq, kOOB);
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(s_base + int64_t(kt) * BK * lds_, kOOB);
        raw[SET][0] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rq, int(in ? q_off : kOOB), 0, 0));
        if constexpr (DW)
            raw[SET][1] = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rq, int(in && b_in2 ? q_off + 16 : kOOB), 0, 0));
        raw_scale[SET] = __builtin_amdgcn_raw_buffer_load_b8(rs, int(in ? s_off : kOOB), 0, 0);
    };
    const int b_wo = b_blk * REGION + b_row * 64, b_flip = (b_blk >> 2) & 1;
    // Chunk t (eight columns) of the thread's block, converted and written.
    auto write_b = [&](auto set_c, auto buf_c, auto t_c) __attribute__((always_inline)) {
        constexpr int SET = decltype(set_c)::value, T = decltype(t_c)::value;
        uint8_t *const dst = decltype(buf_c)::value ? b_lds1 : b_lds0;
        u32x4_t v;
        if constexpr (DW) {
            const float s = mx_scale(raw_scale[SET]);
            const u32x2_t lo = mx8_to_bf16(raw[SET][T / 2][2 * (T & 1)], s), hi = mx8_to_bf16(raw[SET][T / 2][2 * (T & 1) + 1], s);
            v = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
        } else {
            v = mx4_to_bf16(raw[SET][0][T], mx4_scale(raw_scale[SET]));
        }
        *reinterpret_cast<u32x4_t *>(dst + b_wo + 16 * (T ^ b_flip)) = v;
    };

    // ---- fragments
    const int frag_row = lane & 31, half = lane >> 5;
    const int wrow0 = wave_m * (BM / WM), wcol0 = wave_n * (BN / WN);
    const int r0 = wrow0 + frag_row;
    const int grp = lane >> 4, g16 = lane & 15;
    const int tr_row = g16 >> 2, tr_k = (grp >> 1) * 8 + tr_row;      // row of a transpose read, in the k-step
    int a_fo[DW ? TM : 2][4];
    if constexpr (DW) {
        const int bz = ring_bswz<DT_BF16, A_CPR>(tr_row);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int colb = (wrow0 + 32 * i) * 2 + (g16 & 3) * 8 + (grp & 1) * 32;
#pragma unroll
            for (int s = 0; s < 4; ++s) a_fo[i][s] = (64 * group + 16 * s + tr_k) * A_PITCH + (((colb >> 4) ^ bz) << 4) + (colb & 15);
        }
    } else {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int s = 0; s < 4; ++s) a_fo[p][s] = group * A_PART + r0 * 128 + 16 * (swz(2 * s + half, r0) ^ (4 * p));
    }
    int b_fo[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int blk = wcol0 / 32 + j;
        b_fo[j] = blk * REGION + (64 * group + tr_k) * 64 + 16 * ((2 * (grp & 1) + ((g16 & 3) >> 1)) ^ ((blk >> 2) & 1)) + 8 * (g16 & 1);
    }
    u32x4_t fa[2][TM], fb[2][TN];
    auto load_frags = [&](const uint8_t *as, auto buf_c, auto s_c, auto slot_c) __attribute__((always_inline)) {
        constexpr int S = decltype(s_c)::value, SLOT = decltype(slot_c)::value;
        const uint8_t *const bs = decltype(buf_c)::value ? b_lds1 : b_lds0;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if constexpr (DW) {
                const u32x2_t lo = lds_read_tr<DT_BF16>(as + a_fo[i][S]), hi = lds_read_tr<DT_BF16>(as + a_fo[i][S] + 4 * A_PITCH);
                fa[SLOT][i] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
            } else {
                fa[SLOT][i] = *reinterpret_cast<const u32x4_t *>(as + a_fo[i & 1][S] + 4096 * i);
            }
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const u32x2_t lo = lds_read_tr<DT_BF16>(bs + b_fo[j] + S * 1024), hi = lds_read_tr<DT_BF16>(bs + b_fo[j] + S * 1024 + 256);
            fb[SLOT][j] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
        }
    };
    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[1][i] = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[1][j] = u32x4_t{0u, 0u, 0u, 0u};
    auto multiply = [&](auto slot_c) __attribute__((always_inline)) {
        constexpr int SLOT = decltype(slot_c)::value;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = mfma32<DT_BF16>(fa[SLOT][i], fb[SLOT][j], acc[i][j]);
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;

    // K ends inside a chunk of A's rows: what follows it is not part of the sum.
    auto cut_a = [&](int kt, uint8_t *as) __attribute__((always_inline)) {
        if constexpr (!DW) {
            if (kt != nk - 1 || (k_len & 7) == 0) return;
            const int kl = k_len - kt * BK, part = kl / 64, c = kl % 64 / 8;
            for (int r = tid; r < BM; r += THREADS)
                for (int e = kl & 7; e < 8; ++e) reinterpret_cast<uint16_t *>(as + part * A_PART + r * 128 + 16 * swz(c, r))[e] = 0;
            phase_barrier();
        }
    };
    // One stage: buffers BUF hold stage kt, set 1 - BUF the codes of stage kt + 1.  On entry
    // slot 1 holds the fragments of the stage before's last k-step, whose MFMAs run under the
    // latency of this stage's first reads.
    auto stage = [&](int kt, auto buf_c) __attribute__((always_inline)) {
        constexpr int BUF = decltype(buf_c)::value;
        using OTHER = std::integral_constant<int, 1 - BUF>;
        const uint8_t *const as = a_lds[BUF];
        cut_a(kt, a_lds[BUF]);
        // The codes of stage kt + 1 have arrived (loaded a stage ago): said here, before the
        // loads below, so that their use does not wait for those.
#pragma unroll
        for (int i = 0; i < CODES / 16; ++i) asm volatile("" : "+v"(raw[1 - BUF][i]));
        asm volatile("" : "+v"(raw_scale[1 - BUF]));
        load_a(kt + 1, 1 - BUF);
        load_b(kt + 2, buf_c);
        load_frags(as, buf_c, I0{}, I0{});
        write_b(OTHER{}, OTHER{}, I0{});
        multiply(I1{});
        load_frags(as, buf_c, I1{}, I1{});
        write_b(OTHER{}, OTHER{}, I1{});
        multiply(I0{});
        load_frags(as, buf_c, I2{}, I0{});
        write_b(OTHER{}, OTHER{}, I2{});
        multiply(I1{});
        load_frags(as, buf_c, I3{}, I1{});
        write_b(OTHER{}, OTHER{}, I3{});
        multiply(I0{});
        ring_barrier<RAW>();              // A of stage kt + 1 is in LDS; the codes of kt + 2 may be on their way
    };

    if (nk > 0) {
        load_b(0, I0{});
        load_b(1, I1{});
        load_a(0, 0);
        static_for<0, 4>([&](auto t) { write_b(I0{}, I0{}, t); });
        stage_barrier();
        int kt = 0;
        for (; kt + 1 < nk; kt += 2) {
            stage(kt, I0{});
            stage(kt + 1, I1{});
        }
        if (kt < nk) stage(kt, I0{});
        multiply(I1{});
    }
    stage_barrier();
    mx_sum_groups<WK, BLOCKS * REGION>(acc, b_lds0, group, tid);
    mx_store_tile<BM, BN, TM, TN>(a.g, acc, tm, tn, slice, m0 + wrow0, n0 + wcol0, lane, group == 0, *reinterpret_cast<int *>(a_lds[0]));
}

}  // namespace gemm
