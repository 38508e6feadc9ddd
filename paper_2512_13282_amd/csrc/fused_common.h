// fused_common.h -- device helpers of the feed-forward and adapter kernels: activations, the
// sum over K slices, and the epilogues, which see whole sums in registers.
#pragma once

#include "../../include/ffn_mi355x.h"
#include "fused.h"
#include "mx_common.h"

namespace gemm {

// ---------------------------------------------------------------------------
// act(g) and act'(g) in fp32.  With p = 1 / (1 + e^-z) for silu (z = g) and the tanh form of gelu
// (z = 2 sqrt(2 / pi) (g + 0.044715 g^3), as (1 + tanh(z / 2)) / 2 = p), and p the normal distribution for gelu
// itself, act is g p.  e^x by the hardware's 2^x: the argument's rounding costs |x| 2^-24 of the
// value, far below the bf16 result's half step (2^-8) down to where e^-z passes the range of fp32 and p becomes 0 (act below
// 2^-100).
// ---------------------------------------------------------------------------
template <int ACT>
__device__ __forceinline__ float act_value(float g) {
    if constexpr (ACT == FFN_SILU) {
        return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g));
    } else if constexpr (ACT == FFN_GELU) {
        return 0.5f * g * erfcf(-0.70710678f * g);
    } else if constexpr (ACT == FFN_GELU_TANH) {
        const float c = fminf(fmaxf(g, -16.0f), 16.0f);        // p is 0 or 1 there, and the cube stays finite
        return g * __builtin_amdgcn_rcpf(1.0f + __expf(-1.59576912f * c * (1.0f + 0.044715f * c * c)));
    } else {
        return g < 0.0f ? 0.0f : g;                             // a NaN stays one
    }
}
template <int ACT>
__device__ __forceinline__ void act_both(float g, float &a, float &d) {
    if constexpr (ACT == FFN_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
        a = g * p;
        d = p * (1.0f + g * (1.0f - p));
    } else if constexpr (ACT == FFN_GELU) {
        const float p = 0.5f * erfcf(-0.70710678f * g);
        a = g * p;
        d = p + g * (0.39894228f * __expf(-0.5f * g * g));
    } else if constexpr (ACT == FFN_GELU_TANH) {
        const float c = fminf(fmaxf(g, -16.0f), 16.0f);
        const float p = __builtin_amdgcn_rcpf(1.0f + __expf(-1.59576912f * c * (1.0f + 0.044715f * c * c)));
        a = g * p;
        d = p + g * (p * (1.0f - p)) * (1.59576912f * (1.0f + 0.134145f * c * c));
    } else {
        a = g < 0.0f ? 0.0f : g;
        d = g != g ? g : g > 0.0f ? 1.0f : 0.0f;
    }
}

// Calls f with the activation as a compile-time constant.
template <typename F>
__device__ __forceinline__ void with_act(int act, F &&f) {
    if (act == FFN_SILU) f(std::integral_constant<int, FFN_SILU>{});
    else if (act == FFN_GELU) f(std::integral_constant<int, FFN_GELU>{});
    else if (act == FFN_GELU_TANH) f(std::integral_constant<int, FFN_GELU_TANH>{});
    else f(std::integral_constant<int, FFN_RELU>{});
}

// Four bf16 values of a row from column `col` on: the first `left` of them, zeros after them.
__device__ __forceinline__ u32x2_t load4_bf16(const uint16_t *p, int64_t left) {
    u32x2_t v{0u, 0u};
    if (left >= 4) {
        v = *reinterpret_cast<const u32x2_el_t *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) v[e / 2] |= uint32_t(p[e]) << (16 * (e & 1));
    }
    return v;
}
__device__ __forceinline__ void store4_bf16(uint16_t *p, int64_t left, uint32_t lo, uint32_t hi) {
    if (left >= 4) {
        *reinterpret_cast<u32x2_el_t *>(p) = u32x2_t{lo, hi};
    } else {
        if (left > 0) p[0] = uint16_t(lo);
        if (left > 1) p[1] = uint16_t(lo >> 16);
        if (left > 2) p[2] = uint16_t(hi);
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return uint32_t(bf16_nearest_even(lo)) | (uint32_t(bf16_nearest_even(hi)) << 16);
}

// ---------------------------------------------------------------------------
// A wave's fragments: TM x TN of 32 x 32, TN / 2 in each half of the tile's columns.  Fragment (i, j) starts at
// row r0 + 32 i and column c0 + 32 (j % (TN / 2)) + HALF (j / (TN / 2)).
//
// GATED: the first half's sums are G's, the second's U's at the same places: c0 and N count columns of H.
// The products are rounded once, H from the fp32 sums; G and U (where kept) ride through
// the quad's transpose as a pair of bf16 in one register.
// ---------------------------------------------------------------------------
template <int ACT, bool KEEP, int TM, int TN>
__device__ __forceinline__ void store_gated_as(const FusedArgs &a, const f32x16_t (&acc)[TM][TN], int64_t r0, int64_t c0, int lane) {
    const int64_t row0 = r0 + 4 * (lane >> 5) + (lane & 3);
    const int64_t rows_left = a.g.M - row0;
    uint16_t *const h = static_cast<uint16_t *>(a.g.C), *const gs = static_cast<uint16_t *>(a.C2), *const us = static_cast<uint16_t *>(a.C3);
#pragma unroll
    for (int j = 0; j < TN / 2; ++j) {
        const int64_t col = c0 + (lane & 28) + 32 * j, left = a.g.N - col;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t x[4], y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float g = acc[i][j][4 * q + k], u = acc[i][j + TN / 2][4 * q + k];
                    x[k] = __builtin_bit_cast(uint32_t, act_value<ACT>(g) * u);
                    if constexpr (KEEP) y[k] = pack_bf16(g, u);
                }
                quad_transpose(x, lane);
                if constexpr (KEEP) quad_transpose(y, lane);
                const int dr = 32 * i + 8 * q;
                if (dr < rows_left) {
                    auto f = [](uint32_t v) { return __builtin_bit_cast(float, v); };
                    store4_bf16(h + (row0 + dr) * a.g.ldc + col, left, pack_bf16(f(x[0]), f(x[1])), pack_bf16(f(x[2]), f(x[3])));
                    if constexpr (KEEP) {
                        store4_bf16(gs + (row0 + dr) * a.ldc2 + col, left, perm(y[1], y[0], 0x05040100u), perm(y[3], y[2], 0x05040100u));
                        store4_bf16(us + (row0 + dr) * a.ldc3 + col, left, perm(y[1], y[0], 0x07060302u), perm(y[3], y[2], 0x07060302u));
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}
template <int TM, int TN>
__device__ __forceinline__ void store_gated(const FusedArgs &a, const f32x16_t (&acc)[TM][TN], int64_t r0, int64_t c0, int lane) {
    with_act(a.act, [&](auto act) __attribute__((always_inline)) {
        constexpr int ACT = decltype(act)::value;
        if (a.C2 != nullptr) store_gated_as<ACT, true>(a, acc, r0, c0, lane);
        else store_gated_as<ACT, false>(a, acc, r0, c0, lane);
    });
}

// GRAD: the sums are dH; G and U are read where dG, dU and H are written, the next fragments' ahead of
// this one's stores.  Each result is rounded once, from G and U as they were kept.
template <int ACT, int HALF, int TM, int TN>
__device__ __forceinline__ void store_grad_as(const FusedArgs &a, const f32x16_t (&acc)[TM][TN], int64_t r0, int64_t c0, int lane) {
    const int64_t row0 = r0 + 4 * (lane >> 5) + (lane & 3);
    const int64_t rows_left = a.g.M - row0;
    const uint16_t *const gs = static_cast<const uint16_t *>(a.G), *const us = static_cast<const uint16_t *>(a.U);
    uint16_t *const dg = static_cast<uint16_t *>(a.g.C), *const du = static_cast<uint16_t *>(a.C2), *const h = static_cast<uint16_t *>(a.C3);
    auto column = [&](int j) __attribute__((always_inline)) {
        return c0 + (lane & 28) + 32 * (j % (TN / 2)) + HALF * (j / (TN / 2));
    };
    constexpr int AHEAD = TM * TN <= 4 ? TM * TN : TM * TN <= 6 ? 5 : 4;      // fragments of G and U on their way
    u32x2_t kept[AHEAD][4][2];
    auto fetch = [&](auto f_c) __attribute__((always_inline)) {
        constexpr int F = decltype(f_c)::value, J = F / TM, I = F % TM;
        const int64_t col = column(J), left = a.g.N - col;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int dr = 32 * I + 8 * q;
            kept[F % AHEAD][q][0] = kept[F % AHEAD][q][1] = u32x2_t{0u, 0u};
            if (dr < rows_left) {
                kept[F % AHEAD][q][0] = load4_bf16(gs + (row0 + dr) * a.ldg + col, left);
                kept[F % AHEAD][q][1] = load4_bf16(us + (row0 + dr) * a.ldu + col, left);
            }
        }
    };
    static_for<0, AHEAD>([&](auto f_c) __attribute__((always_inline)) { fetch(f_c); });
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, TM * TN>([&](auto f_c) __attribute__((always_inline)) {
        constexpr int F = decltype(f_c)::value, J = F / TM, I = F % TM;
        const int64_t col = column(J), left = a.g.N - col;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint32_t x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float e = acc[I][J][4 * q + k];
                x[k] = __builtin_bit_cast(uint32_t, e);
            }
            quad_transpose(x, lane);
            float ga[4], ua[4], ha[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float d = __builtin_bit_cast(float, x[k]);
                const float g = bf16_to_f32((kept[F % AHEAD][q][0][k / 2] >> (16 * (k & 1))) & 0xffffu);
                const float u = bf16_to_f32((kept[F % AHEAD][q][1][k / 2] >> (16 * (k & 1))) & 0xffffu);
                float value, slope;
                act_both<ACT>(g, value, slope);
                ga[k] = d * u * slope;
                ua[k] = d * value;
                ha[k] = value * u;
            }
            const int dr = 32 * I + 8 * q;
            if (dr < rows_left) {
                store4_bf16(dg + (row0 + dr) * a.g.ldc + col, left, pack_bf16(ga[0], ga[1]), pack_bf16(ga[2], ga[3]));
                store4_bf16(du + (row0 + dr) * a.ldc2 + col, left, pack_bf16(ua[0], ua[1]), pack_bf16(ua[2], ua[3]));
                if (h != nullptr) store4_bf16(h + (row0 + dr) * a.ldc3 + col, left, pack_bf16(ha[0], ha[1]), pack_bf16(ha[2], ha[3]));
            }
        }
        if constexpr (F + AHEAD < TM * TN) fetch(std::integral_constant<int, F + AHEAD>{});
        __builtin_amdgcn_sched_barrier(0);
    });
}

// The other operators: the sums themselves, as the dense products store them.
template <int WAVES, int HALF, int TM, int TN>
__device__ __forceinline__ void store_plain(const KernelArgs &g, const f32x16_t (&acc)[TM][TN], int64_t r0, int64_t c0, int lane) {
    static_assert(TN == 2, "one fragment in each half");
    if (g.epilogue == EPI_BF16) store_c_direct<DT_BF16, EPI_BF16, WAVES, HALF>(g, acc, r0, c0, lane);
    else store_c_direct<DT_BF16, EPI_NONE, WAVES, HALF>(g, acc, r0, c0, lane);
}

// ---------------------------------------------------------------------------
// What a workgroup computes.  The first `whole` workgroups have an output tile each with all of K.  The rest fill a last
// round that would leave compute units idle: with slices of K of the tiles after those, or (`tail`) with lower tiles over the
// rows or columns after those, which end sooner (gated 2048 x 11008: 512 tiles of 256 rows in two rounds, then 242 of
// 192 rows in place of 176).  As in map_tile, each XCD has a contiguous range of either part, and tiles are walked in
// groups of rows.
// ---------------------------------------------------------------------------
struct FusedWork {
    int64_t m0, n0;              // of the tile
    int which;                   // DW: the second matrix
    int first, count;            // stages of 64 k
    int slot, slice, slices;     // the tile's place among those in slices, this slice of it and how many there are
    bool low;                    // one of the lower tiles
};
constexpr int kEarlyFrom = 128;
template <int BM, int LOW, int COLS>
__device__ __forceinline__ FusedWork fused_work(const FusedArgs &a, int all) {
    const KernelArgs &g = a.g;
    // GRAD: lower tiles also fill the second half of the first round, so that the compute units end their tiles, and read and
    // write ten bytes for each of their elements, at different times from then on (2048 x 11008 x 4096: 204 against the best other
    // plan's 226 us on one card, 224 against 221 on a second, 214 against 233 on a third).
    const int at = int(blockIdx.x), early = LOW > 0 ? a.early : 0;
    const bool rest = (early > 0 && at >= kEarlyFrom && at < kEarlyFrom + early) || at >= a.whole + early;
    const int total = rest ? int(gridDim.x) - a.whole : a.whole;
    const int hw = early == 0 ? (rest ? at - a.whole : at) : rest ? (at < kEarlyFrom + early ? at - kEarlyFrom : at - a.whole) : at < kEarlyFrom ? at : at - early;
    const int per = total / 8, rem = total % 8, xcd = hw % 8, local = hw / 8;
    const int id = xcd < rem ? xcd * (per + 1) + local : rem * (per + 1) + (xcd - rem) * per + local;
    FusedWork w;
    w.low = LOW > 0 && rest;
    const int tiles_m = w.low ? a.tail.tiles_m : g.tiles_m, tiles_n = w.low ? a.tail.tiles_n : g.tiles_n;
    const int sliced = w.low ? 1 : rest ? tiles_m * tiles_n - a.whole : 1;
    w.slice = w.low || !rest ? 0 : id / sliced;
    w.slot = w.low || !rest ? 0 : id % sliced;
    w.slices = w.low || !rest ? 1 : g.split_k;
    const int t = w.low || !rest ? id : a.whole + w.slot;
    const int width = g.group_m * tiles_n, first_m = t / width * g.group_m;
    const int rows = tiles_m - first_m < g.group_m ? tiles_m - first_m : g.group_m;
    const int tm = first_m + t % width % rows, tn = t % width / rows;
    // DW: tile rows from `half` on are the second matrix's (lower tiles over the last rows: all are).
    const int half = w.low ? a.tail.half : a.half;
    w.which = tm >= half;
    const int64_t row0 = w.low ? a.tail.row : 0;
    w.m0 = row0 + int64_t(w.which ? tm - half : tm) * (w.low ? LOW : BM);
    w.n0 = (w.low ? a.tail.col : 0) + int64_t(tn) * COLS;
    const int chunk = int(g.k_chunk / 64);
    w.first = w.slices > 1 ? w.slice * chunk : 0;
    w.count = w.slices > 1 && w.first + chunk < all ? chunk : all - w.first;
    return w;
}

// ---------------------------------------------------------------------------
// K slices: every slice leaves its sums in the workspace as its registers hold them and the one that
// arrives last adds the others' to its own, all in the order of the slices, whichever it is (mx_common.h says how
// the accesses are ordered).  True in every thread of the workgroup that holds the whole sums.
// ---------------------------------------------------------------------------
template <int THREADS, int TM, int TN>
__device__ __forceinline__ bool sum_slices(const KernelArgs &g, f32x16_t (&acc)[TM][TN], int slot, int slice, int slices, int64_t rows, int &flag) {
    constexpr uint32_t SLICE = uint32_t(TM * TN * 16 * 4) * THREADS;
    const __amdgpu_buffer_rsrc_t parts = mx_parts(g, slot, SLICE);
    const uint32_t off = threadIdx.x * 16;
    // Register group q of fragment row i: rows 32 i + 8 q .. + 7 of the wave's; past M nothing is left or fetched.
    auto at = [&](int s, int i, int j, int q) __attribute__((always_inline)) {
        return uint32_t(s) * SLICE + off + uint32_t(((i * TN + j) * 4 + q) * THREADS) * 16;
    };
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (32 * i + 8 * q < rows)
                    mx_store_part(parts, at(slice, i, j, q),
                                  f32x4_t{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
        flag = __hip_atomic_fetch_add(&g.counters[slot], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == unsigned(slices - 1);
    __syncthreads();
    if (flag == 0) return false;
    // ((part 0 + part 1) + ...) + own + ... : own stays in its registers, what comes before it is added up beside them.
    // FRAGMENTS fragments of WAYS slices on the way at once, as many registers as a tile of that size leaves.
    constexpr int F = TM * TN;
    auto pass = [&](auto f0_c, auto count_c, auto ways_c, int begin, int end, auto &&into) __attribute__((always_inline)) {
        constexpr int F0 = decltype(f0_c)::value, COUNT = decltype(count_c)::value, WAYS = decltype(ways_c)::value;
#pragma unroll 1
        for (int s = begin; s < end; s += WAYS) {
            f32x4_t v[WAYS][COUNT][4];
#pragma unroll
            for (int u = 0; u < WAYS; ++u)
#pragma unroll
                for (int f = 0; f < COUNT; ++f)
#pragma unroll
                    for (int q = 0; q < 4; ++q)              // past the end zeros, which change nothing
                        v[u][f][q] = mx_load_part(parts, s + u < end && 32 * ((F0 + f) / TN) + 8 * q < rows ? at(s + u, (F0 + f) / TN, (F0 + f) % TN, q) : kOOB);
#pragma unroll
            for (int u = 0; u < WAYS; ++u)
#pragma unroll
                for (int f = 0; f < COUNT; ++f)
#pragma unroll
                    for (int q = 0; q < 4; ++q) into(f, q, v[u][f][q]);
        }
    };
    auto group = [&](auto f0_c, auto count_c, auto ways_c) __attribute__((always_inline)) {
        constexpr int F0 = decltype(f0_c)::value, COUNT = decltype(count_c)::value;
        auto add = [&](int f, int q, f32x4_t v) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[(F0 + f) / TN][(F0 + f) % TN][4 * q + e] += v[e];
        };
        if (slice > 1) {
            f32x4_t sum[COUNT][4] = {};
            pass(f0_c, count_c, ways_c, 0, slice, [&](int f, int q, f32x4_t v) __attribute__((always_inline)) { sum[f][q] += v; });
#pragma unroll
            for (int f = 0; f < COUNT; ++f)
#pragma unroll
                for (int q = 0; q < 4; ++q) add(f, q, sum[f][q]);
        } else {
            pass(f0_c, count_c, std::integral_constant<int, 1>{}, 0, slice, add);
        }
        pass(f0_c, count_c, ways_c, slice + 1, slices, add);
    };
    constexpr int FRAGMENTS = F <= 4 ? F : 2, WAYS = F <= 2 ? 4 : 1;
    static_assert(F % FRAGMENTS == 0, "whole groups");
    static_for<0, F / FRAGMENTS>([&](auto k) __attribute__((always_inline)) {
        group(std::integral_constant<int, decltype(k)::value * FRAGMENTS>{}, std::integral_constant<int, FRAGMENTS>{},
              std::integral_constant<int, WAYS>{});
        if constexpr (F > 4) __builtin_amdgcn_sched_barrier(0);
    });
    mx_reset_counter(g, slot);
    return true;
}

}  // namespace gemm
