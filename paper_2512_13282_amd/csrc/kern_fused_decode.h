// kern_fused_decode.h -- the gated product and the projection with adapters for few rows: a read of the weights.
#pragma once

#include "fused_expand.h"
#include "kern_mx_decode.h"

namespace gemm {

constexpr int kFewRanks = 64;        // ranks of h in LDS at a time
// Threads to an output of the adapters' part: 16 columns of 16 MT tokens, KW waves.
constexpr int few_rows_share(int MT, int KW) { return 64 * KW / (256 * MT) > 0 ? 64 * KW / (256 * MT) : 1; }

// The adapters' part of a tile of 16 columns from n0 on: h's planes are summed into LDS and each output takes its
// h . B_i row on the vector unit, in fp32, while the first weights are on their way.
template <int MT, int KW, int S, int T>
__device__ __forceinline__ void few_rows_adapters(const FusedArgs &a, float (&hs)[T][kFewRanks + 4], float (&extra)[S][T][16], int64_t n0, int tid) {
    constexpr int THREADS = 64 * KW, TOKENS = 16 * MT, SHARE = few_rows_share(MT, KW);
    constexpr int OUTS = (16 * TOKENS * SHARE + THREADS - 1) / THREADS;                   // outputs to a thread
    const int64_t M = a.g.M, N = a.g.N;
    float sum[OUTS] = {};
    const int r = a.n > 0 ? a.r : 0;
    for (int j0 = 0; j0 < r; j0 += kFewRanks) {
        const int ranks = r - j0 < kFewRanks ? r - j0 : kFewRanks;
        for (int i = tid; i < TOKENS * kFewRanks; i += THREADS) {
            const int t = i / kFewRanks, j = i % kFewRanks;
            float v = 0.0f;
            if (t < M && j < ranks) {
                float parts[8];                                           // all of them on the way at once
#pragma unroll
                for (int p = 0; p < 8; ++p) parts[p] = p < a.planes ? a.h[p * a.h_plane + int64_t(t) * a.r + j0 + j] : 0.0f;
#pragma unroll
                for (int p = 0; p < 8; ++p) v += parts[p];
            }
            hs[t][j] = v;
        }
        phase_barrier();
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
            const int i = tid + o * THREADS, at = i % (16 * TOKENS), share = i / (16 * TOKENS);
            const int t = at >> 4, c = at & 15;
            const int own = t < M ? a.index[t] : -1;
            if (uint32_t(own) >= uint32_t(a.n) || n0 + c >= N) continue;
            const uint16_t *const q = static_cast<const uint16_t *>(a.Q) + own * a.sq + (n0 + c) * a.ldq + j0;
            for (int j = 8 * share; j < ranks; j += 8 * SHARE) {
                const u32x4_t v = load8_bf16(q + j, ranks - j);
#pragma unroll
                for (int e = 0; e < 8; ++e) {                         // past the rank hs and v are zeros
                    const float b = __builtin_bit_cast(float, e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
                    sum[o] += hs[t][j + e] * b;
                }
            }
        }
        phase_barrier();
    }
#pragma unroll
    for (int o = 0; o < OUTS; ++o) {
        const int i = tid + o * THREADS, at = i % (16 * TOKENS);
        if (i < 16 * TOKENS * SHARE) extra[i / (16 * TOKENS)][at >> 4][at & 15] = sum[o];
    }
}

// The waves' sums, added up in their order, with the adapters' part and the epilogue: wave m has tokens 16 m .. + 15.
template <int OP, int MT, int KW, int S, int T>
__device__ __forceinline__ void few_rows_store(const FusedArgs &a, const f32x4_t (&part)[KW][MT][64], const float (&extra)[S][T][16], int64_t n0,
                                               int wave, int lane) {
    constexpr int SHARE = few_rows_share(MT, KW);
    const int l16 = lane & 15, grp = lane >> 4;
    const int64_t M = a.g.M, N = a.g.N;
    if (wave >= MT) return;
    auto total = [&](int l) __attribute__((always_inline)) {
        f32x4_t s = part[0][wave][l];
#pragma unroll
        for (int k = 1; k < KW; ++k) s += part[k][wave][l];
        return s;
    };
    const int64_t t = 16 * wave + l16;
    if constexpr (OP == FUSED_GATED) {
        if (grp >= 2) return;
        const f32x4_t g = total(lane), u = total(lane + 32);
        const int64_t col = n0 + 4 * grp, left = t < M ? N - col : 0;
        if (left <= 0) return;
        with_act(a.act, [&](auto act) __attribute__((always_inline)) {
            constexpr int ACT = decltype(act)::value;
            float h[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = act_value<ACT>(g[e]) * u[e];
            store4_bf16(static_cast<uint16_t *>(a.g.C) + t * a.g.ldc + col, left, pack_bf16(h[0], h[1]), pack_bf16(h[2], h[3]));
        });
        if (a.C2 != nullptr) {
            store4_bf16(static_cast<uint16_t *>(a.C2) + t * a.ldc2 + col, left, pack_bf16(g[0], g[1]), pack_bf16(g[2], g[3]));
            store4_bf16(static_cast<uint16_t *>(a.C3) + t * a.ldc3 + col, left, pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]));
        }
    } else {
        f32x4_t s = total(lane);
        const int64_t col = n0 + 4 * grp;
#pragma unroll
        for (int k = 0; k < SHARE; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += extra[k][16 * wave + l16][4 * grp + e];
        if (t < M && col < N) mx_store4(a.g, t, col, s);
    }
}

// ---------------------------------------------------------------------------
// Up to 16 MT rows of A.  A workgroup holds 16 rows of weights (ADAPT: 16 columns of C; GATED: eight of the one and the
// same eight of the other) and the whole of K, of which its KW waves take contiguous parts.  Weights and A go from memory
// to registers, U chunks of 64 k on the way per wave: lane l loads 16 bytes of row l % 16 at k = 8 (l / 16) of each
// half of a chunk, its share of one 16 x 16 x 32 MFMA, so that the two loads together use whole 128-byte lines.  No
// element of either is used by two waves, so nothing passes through LDS but the waves' sums, added up in a fixed
// order.  Output register e of lane l is weight row 4 (l / 16) + e of token l % 16.  Operands may lie at any address.
//
// Bound by the read of the weights for one row (gated 1 x 14336 x 4096, 235 MB: 39.3 us; the tile kernel 45.1), by the
// latency of a few trips to memory for small odd sizes (37 x 2051 x 2049: 20.8 us; copied to aligned rows for the tile
// kernel 21.5).  A's pieces pass the load path like the weights': 16 rows cost 1 x 4096 x 14336's 34 us another 16, and
// fused_stream_kernel or the tile kernel takes those where rows are aligned.
// ---------------------------------------------------------------------------
template <int OP, int MT, int KW, int U, bool ODD>
__global__ __launch_bounds__(64 * KW) void fused_decode_kernel(FusedArgs a) {
    static_assert(OP == FUSED_GATED || OP == FUSED_ADAPT, "weights stored N x K");
    constexpr bool EXPAND = OP == FUSED_ADAPT;
    constexpr int TOKENS = 16 * MT;
    __shared__ __attribute__((aligned(16))) f32x4_t part[KW][MT][64];
    __shared__ float hs[EXPAND ? TOKENS : 1][kFewRanks + 4];
    __shared__ float extra[few_rows_share(MT, KW)][EXPAND ? TOKENS : 1][16];

    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    const int64_t M = a.g.M, N = a.g.N, K = a.g.K;
    const int64_t n0 = int64_t(blockIdx.x) * (OP == FUSED_GATED ? 8 : 16);

    const int64_t chunks = (K + 63) / 64, whole = K / 64, per = (chunks + KW - 1) / KW;
    const int64_t c0 = wave * per, c1 = c0 + per < chunks ? c0 + per : chunks;
    const int n = int((c1 < whole ? c1 : whole) - c0);                    // whole chunks; <= 0 for a wave without any

    // A row past the end reads the last one; its results are not stored.
    const uint16_t *wp;
    if constexpr (OP == FUSED_GATED) {
        const int64_t row = n0 + (l16 & 7) < N ? n0 + (l16 & 7) : N - 1;
        wp = l16 < 8 ? static_cast<const uint16_t *>(a.g.B) + row * a.g.ldb : static_cast<const uint16_t *>(a.B2) + row * a.ldb2;
    } else {
        const int64_t row = n0 + l16 < N ? n0 + l16 : N - 1;
        wp = static_cast<const uint16_t *>(a.g.B) + row * a.g.ldb;
    }
    wp += c0 * 64 + 8 * grp;
    const uint16_t *xp[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t t = 16 * m + l16 < M ? 16 * m + l16 : M - 1;
        xp[m] = static_cast<const uint16_t *>(a.g.A) + t * a.g.lda + c0 * 64 + 8 * grp;
    }
    u32x4_t w[U][2], x[U][MT][2];
    auto load = [&](int u, int c) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            w[u][p] = load8_any<ODD>(wp + int64_t(c) * 64 + 32 * p);
#pragma unroll
            for (int m = 0; m < MT; ++m) x[u][m][p] = load8_any<ODD>(xp[m] + int64_t(c) * 64 + 32 * p);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n) load(u, u);

    if constexpr (EXPAND) few_rows_adapters<MT, KW>(a, hs, extra, n0, tid);

    f32x4_t acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int u) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m] = mfma16_bf16(w[u][p], x[u][m][p], acc[m]);
    };
    int i = 0;
    for (; i + 2 * U <= n; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            multiply(u);
            load(u, i + U + u);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (i + u < n) multiply(u);
        if (i + U + u < n) load(u, i + U + u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (i + U + u < n) multiply(u);
    if (chunks > whole && whole >= c0 && whole < c1) {                    // the end of K that is no whole chunk
        const int c = int(whole - c0);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int64_t left = K - whole * 64 - 32 * p - 8 * grp;
            w[0][p] = load8_bf16(wp + int64_t(c) * 64 + 32 * p, left);
#pragma unroll
            for (int m = 0; m < MT; ++m) x[0][m][p] = load8_bf16(xp[m] + int64_t(c) * 64 + 32 * p, left);
        }
        multiply(0);
    }

#pragma unroll
    for (int m = 0; m < MT; ++m) part[wave][m][lane] = acc[m];
    __syncthreads();
    few_rows_store<OP, MT, KW>(a, part, extra, n0, wave, lane);
}

// ---------------------------------------------------------------------------
// The same tiles for operands on 16-byte rows.  Each wave streams its part of K through NS stages of LDS of its own, 64 k
// of 16 rows of weights and 16 MT of A each, with direct-to-LDS loads of whole 128-byte row pieces: 64-byte pieces straight
// into registers, as above, cost the load path nearly twice the time once A has more than a few rows.  A wave waits
// for its own loads only; nothing is shared, so there is no barrier before the sums.  Rows of A past M are
// not read (zeros).
//
// Measured: adapters 16 x 4096 x 14336 (117 MB of weights, and as many bytes of A through the compute units' load paths)
// 27.6 us, with the first product's launch 35.6; fused_decode_kernel in its place 43.6, the tile kernel in twelve slices 43.6.
// For one row the registers win (39.2 against 48.1 us at gated 1 x 14336 x 4096).
// ---------------------------------------------------------------------------
template <int OP, int MT, int KW, int NS>
__global__ __launch_bounds__(64 * KW) void fused_stream_kernel(FusedArgs a) {
    static_assert(OP == FUSED_GATED || OP == FUSED_ADAPT, "weights stored N x K");
    constexpr bool EXPAND = OP == FUSED_ADAPT;
    constexpr int TOKENS = 16 * MT, STAGE = 2048 * (1 + MT), LPS = 2 + 2 * MT;
    static_assert(NS >= 2 && (NS - 1) * LPS < 64, "loads in flight must fit vmcnt");
    __shared__ __attribute__((aligned(1024))) uint8_t ring[KW][NS][STAGE];
    __shared__ __attribute__((aligned(16))) f32x4_t part[KW][MT][64];
    __shared__ float hs[EXPAND ? TOKENS : 1][kFewRanks + 4];
    __shared__ float extra[few_rows_share(MT, KW)][EXPAND ? TOKENS : 1][16];

    const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    const int64_t M = a.g.M, N = a.g.N;
    const int K = int(a.g.K);
    const int64_t n0 = int64_t(blockIdx.x) * (OP == FUSED_GATED ? 8 : 16);
    const int stages = (K + 63) / 64, per = (stages + KW - 1) / KW;
    const int s0 = wave * per, ns = (s0 + per < stages ? s0 + per : stages) - s0;        // <= 0 for a wave without any

    // Loads of a stage: rows 8 i + lane / 8 of the weights (i = 0, 1) and of A (i - 2), 128 bytes each.
    const int lda_b = int(a.g.lda) * 2, ldb_b = int(a.g.ldb) * 2, ldb2_b = int(a.ldb2) * 2;
    const int valid = N - n0 < (OP == FUSED_GATED ? 8 : 16) ? int(N - n0) : (OP == FUSED_GATED ? 8 : 16);
    const uint8_t *const w_base = static_cast<const uint8_t *>(a.g.B) + n0 * ldb_b;
    const uint8_t *const w2_base = OP == FUSED_GATED ? static_cast<const uint8_t *>(a.B2) + n0 * ldb2_b : w_base;
    const uint8_t *const x_base = static_cast<const uint8_t *>(a.g.A);
    const uint32_t w_bytes = uint32_t(valid * ldb_b), w2_bytes = OP == FUSED_GATED ? uint32_t(valid * ldb2_b) : w_bytes, x_bytes = uint32_t(int(M) * lda_b);
    uint32_t voff[LPS];
    int chunk[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = 8 * i + (lane >> 3);
        chunk[i] = swz(lane & 7, row);                                    // of rows 16 further down too
        voff[i] = OP == FUSED_GATED ? uint32_t((lane >> 3) * (i ? ldb2_b : ldb_b) + chunk[i] * 16) : uint32_t(row * ldb_b + chunk[i] * 16);
#pragma unroll
        for (int m = 0; m < MT; ++m) voff[2 + 2 * m + i] = uint32_t((16 * m + row) * lda_b + chunk[i] * 16);
    }
    auto load = [&](int s, auto slot_c) __attribute__((always_inline)) {
        constexpr int SLOT = decltype(slot_c)::value;
        const int rem = s < ns ? K - (s0 + s) * 64 : 0;
        const int64_t at = int64_t(s0 + s) * 128;
        const uint32_t dst = lds_addr(ring[0][0]) + uint32_t(wave * (NS * STAGE) + SLOT * STAGE);
        const i32x4_t rw = ring_rsrc(uniform(w_base + at), uniform(rem > 0 ? w_bytes : 0u));
        const i32x4_t rw2 = ring_rsrc(uniform(w2_base + at), uniform(rem > 0 ? w2_bytes : 0u));
        const i32x4_t rx = ring_rsrc(uniform(x_base + at), uniform(rem > 0 ? x_bytes : 0u));
#pragma unroll
        for (int i = 0; i < LPS; ++i)
            ring_load16(i == 0 ? rw : i == 1 ? rw2 : rx, dst + i * 1024, chunk[i & 1] * 8 < rem ? voff[i] : kOOB);
    };
    if (ns > 0) static_for<0, NS - 1>([&](auto s) { load(decltype(s)::value, s); });

    if constexpr (EXPAND) few_rows_adapters<MT, KW>(a, hs, extra, n0, tid);

    f32x4_t acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    int fo[2];                                                            // k-step p of row l16
#pragma unroll
    for (int p = 0; p < 2; ++p) fo[p] = l16 * 128 + 16 * swz(4 * p + grp, l16);
    if (ns > 0) {
        for (int s = 0; s < ns; s += NS) {
            static_for<0, NS>([&](auto u) __attribute__((always_inline)) {
                constexpr int SLOT = decltype(u)::value;
                if (s + SLOT >= ns) return;
                // This stage has landed, and the reads of the one before it, whose slot the next loads fill, are done.
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * LPS) : "memory");
                load(s + SLOT + NS - 1, std::integral_constant<int, (SLOT + NS - 1) % NS>{});
                const uint8_t *const p0 = ring[wave][SLOT];
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const u32x4_t w = *reinterpret_cast<const u32x4_t *>(p0 + fo[p]);
#pragma unroll
                    for (int m = 0; m < MT; ++m) acc[m] = mfma16_bf16(w, *reinterpret_cast<const u32x4_t *>(p0 + 2048 * (1 + m) + fo[p]), acc[m]);
                }
            });
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                  // the loads past the end
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) part[wave][m][lane] = acc[m];
    __syncthreads();
    few_rows_store<OP, MT, KW>(a, part, extra, n0, wave, lane);
}

}  // namespace gemm
