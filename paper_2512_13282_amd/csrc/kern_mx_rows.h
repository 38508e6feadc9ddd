// kern_mx_rows.h -- C = A . W and C = A^T . X for few rows of C: operands transposed in registers.
#pragma once

#include "kern_mx_decode.h"

namespace gemm {

// ---------------------------------------------------------------------------
// A workgroup holds 128 columns of C, 16 MT rows and one of S slices of K.  Its KW waves take
// contiguous parts of the slice and add their sums up in LDS.  B is W, 4-bit (MX_DX), or X, 8-bit
// (MX_DW); its blocks lie along N, across the sum.
//
// mx_grad_kernel writes every converted value to LDS and reads it back transposed, however few
// rows it then multiplies: 0.88 us per 256 k of a 32 x 64 tile, with loads two or four stages ahead
// alike.  Here the operands go from memory into the registers that the matrix instruction reads, U
// steps of 32 k on the way per wave, and LDS holds nothing but the sums at the end.
//
// Lane l (i = l % 16, g = l / 16) loads columns 8 i .. 8 i + 7 of B's rows 8 g .. 8 g + 7, converts a
// row's codes under the row's scale, and puts pairs of rows together with v_perm: fragment j has
// column 8 i + j at i, and k = 8 g + 0..7 as the 16 x 16 x 32 MFMA wants them.  Of A, DX's fragments lie
// so in memory; DW's come from a dword (two columns of A, rows of C) of each of eight rows
// in the same way, so fragment f has row 2 i + f.  A row has one scale byte per four lanes; each of them loads
// two rows' and quad permutations hand them round.  Output register r of lane l in fragment j is
// column 32 g + 8 r + j of the row at l % 16.
//
// Bound by latencies one after the other: launch, first loads, the sum in LDS, and where K is
// split the slices' sum (2.5 + 1 + 1 + 4 us of the smaller ones), the load path between them.  DX, against
// the best of mx_grad_kernel: 1 x 4096 x 4096 7.3 us (10.1), 16 x 4096 x 4096 8.0 (10.3), 16 x 14336 x
// 4096 12.6 (17.4), 96 x 4096 x 4096 13.2 (17.6), 256 x 4096 x 4096 18.5 (24.2).  DW: 16 x 4096 x 2048
// 8.3 (9.4), 4096 x 16 x 2048 10.7 (10.8), 64 x 4096 x 2048 9.6 (11.5), 16 x 14336 x 4096 15.8 (22.2).
// Pieces of 64 bytes leave half of each 128-byte line that the load path moves unused; W through
// LDS in 16-byte pieces, in the same rows, took 8 to 10 per cent longer.
//
// U and the waves per SIMD by registers: 16 rows and DW leave room for two workgroups per compute unit
// (against U = 3 in one, 16 x 14336 x 4096: 13.3; DW 64 x 4096 x 2048 10.1 with U = 2), 32 and 48 rows
// would spill.  64 rows (16 MT) were never the best.
// ---------------------------------------------------------------------------
template <int OP, int MT, int KW, int U, int WAVES_PER_EU>
__global__ __attribute__((amdgpu_flat_work_group_size(64 * KW, 64 * KW),
                          amdgpu_waves_per_eu(WAVES_PER_EU, WAVES_PER_EU)))
void mx_rows_kernel(MxArgs a) {
    constexpr bool DW = OP == MX_DW;
    constexpr int CODES = DW ? 2 : 1;                        // dwords of a lane's eight codes
    static_assert(KW == 8, "the sum's 512 threads hold four results of each 16 x 128 part");
    static_assert(!DW || MT == 2, "a lane's dword of a row of A is two rows of C");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[KW * 8192];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    int tm, tn, slice;
    map_tile(a.g, tm, tn, slice);
    const int64_t M = a.g.M, N = a.g.N, K = a.g.K;
    const int64_t m0 = int64_t(tm) * 16 * MT, n0 = int64_t(tn) * 128;
    const int64_t lda_b = a.g.lda * 2, ldq = a.g.ldb, lds_ = a.ld_scales;

    // This wave's steps.
    const int64_t k_begin = int64_t(slice) * a.g.k_chunk;
    const int64_t k_end = k_begin + a.g.k_chunk < K ? k_begin + a.g.k_chunk : K;
    const int steps = int((k_end - k_begin + 31) / 32), per = (steps + KW - 1) / KW;
    const int64_t k0 = k_begin + int64_t(wave) * per * 32;
    const int mine = steps - wave * per < per ? steps - wave * per : per;   // <= 0 for a wave without any
    const bool cut = (k_end - k_begin) % 32 != 0 && mine > 0 && wave * per + mine == steps;
    const int n = cut ? mine - 1 : mine;                     // whole steps; where K ends in a step, that comes last

    // Offsets within a step.  Lanes past N load nothing, and of the step that K ends in neither do rows
    // past it (their codes and scales: zeros).  A may lie at any address, so every load of it stays
    // inside its rows: rows of C past M take the last one's, and are not stored.
    const bool in = n0 + 8 * l16 < N;
    uint32_t w_off[DW ? 1 : 8], s_off[2], a_off[DW ? 1 : MT];
    // DW, short of registers, moves the base from row to row instead.
#pragma unroll
    for (int i = 0; i < (DW ? 1 : 8); ++i) w_off[i] = in ? uint32_t((8 * grp + i) * ldq + 4 * CODES * l16) : kOOB;
#pragma unroll
    for (int i = 0; i < 2; ++i)                              // of the quad's block
        s_off[i] = n0 + 8 * (l16 & 12) < N ? uint32_t((8 * grp + 2 * (lane & 3) + i) * lds_ + l16 / 4) : kOOB;
    const int64_t a_last = M >= 2 ? M - 2 : 0, a_col = m0 < a_last ? m0 : a_last;      // DW: the last dword of A's rows
    if constexpr (DW) {
        a_off[0] = uint32_t(8 * grp * lda_b + 2 * ((m0 + 2 * l16 < a_last ? m0 + 2 * l16 : a_last) - a_col));
    } else {
#pragma unroll
        for (int m = 0; m < MT; ++m) a_off[m] = uint32_t((m0 + 16 * m + l16 < M ? 16 * m + l16 : M - 1 - m0) * lda_b + 16 * grp);
    }
    const uint8_t *const w_base = static_cast<const uint8_t *>(a.g.B) + k0 * ldq + (DW ? n0 : n0 / 2);
    const uint8_t *const s_base = a.scales + k0 * lds_ + n0 / kMxBlock;
    const uint8_t *const a_base = static_cast<const uint8_t *>(a.g.A) + (DW ? k0 * lda_b + a_col * 2 : m0 * lda_b + k0 * 2);

    uint32_t w[U][8][CODES], sc[U][2];
    uint32_t af[U][DW ? 8 : 4 * MT];                         // DX: fragments; DW: dwords of eight rows
    auto load_b = [&](int u, int c, int rows) __attribute__((always_inline)) {
        // A row of the step ends before the next begins: rows past the step's are out of range.
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(s_base + int64_t(c) * 32 * lds_, uint32_t(rows * lds_));
#pragma unroll
        for (int i = 0; i < 2; ++i) sc[u][i] = __builtin_amdgcn_raw_buffer_load_b8(rs, int(s_off[i]), 0, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DW) {
                const __amdgpu_buffer_rsrc_t rw = make_rsrc(w_base + (int64_t(c) * 32 + i) * ldq, uint32_t(rows > i ? (rows - i) * ldq : 0));
                const u32x2_t x = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_raw_buffer_load_b64(rw, int(w_off[0]), 0, 0));
                w[u][i][0] = x[0];
                w[u][i][1] = x[1];
            } else {
                const __amdgpu_buffer_rsrc_t rw = make_rsrc(w_base + int64_t(c) * 32 * ldq, uint32_t(rows * ldq));
                w[u][i][0] = __builtin_amdgcn_raw_buffer_load_b32(rw, int(w_off[i]), 0, 0);
            }
        }
    };
    auto load = [&](int u, int c) __attribute__((always_inline)) {
        load_b(u, c, 32);
        const uint8_t *const p = a_base + int64_t(c) * (DW ? 32 * lda_b : 64);
        if constexpr (DW) {
#pragma unroll
            for (int i = 0; i < 8; ++i) af[u][i] = *reinterpret_cast<const u32_any_mx *>(p + i * lda_b + a_off[0]);
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const u32x4_t x = *reinterpret_cast<const u32x4_any_mx *>(p + a_off[m]);
#pragma unroll
                for (int d = 0; d < 4; ++d) af[u][4 * m + d] = x[d];
            }
        }
    };
    // The step that K ends in, after `rows` of its 32: zeros past them.
    auto load_cut = [&](int c, int rows) __attribute__((always_inline)) {
        load_b(0, c, rows);
        const uint8_t *const p = a_base + int64_t(c) * (DW ? 32 * lda_b : 64);
        if constexpr (DW) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int past = 8 * grp + i - (rows - 1);
                const uint32_t x = *reinterpret_cast<const u32_any_mx *>(p + int64_t(a_off[0]) + (i - (past > 0 ? past : 0)) * lda_b);
                af[0][i] = past > 0 ? 0u : x;
            }
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                uint32_t x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = 8 * grp + e < rows ? e : rows - 1 - 8 * grp;      // may be before this lane's
                    x[e] = *reinterpret_cast<const uint16_t *>(p + int64_t(a_off[m]) + 2 * k);
                }
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    af[0][4 * m + d] = (8 * grp + 2 * d < rows ? x[2 * d] : 0u) | (8 * grp + 2 * d + 1 < rows ? x[2 * d + 1] << 16 : 0u);
            }
        }
    };
    // The lower or upper halves of eight rows' dwords, as the matrix instruction takes eight k.
    auto pairs = [&](const uint32_t (&v)[8], int half) __attribute__((always_inline)) {
        const uint32_t sel = half ? 0x07060302u : 0x05040100u;
        return u32x4_t{perm(v[1], v[0], sel), perm(v[3], v[2], sel), perm(v[5], v[4], sel), perm(v[7], v[6], sel)};
    };
    // The halves of A's dwords (DW) that hold rows 2 i and 2 i + 1 of C: the row at the end of an odd M lies
    // in the upper one, for its dword ends with it.
    const uint32_t a_sel[2] = {DW && m0 + 2 * l16 == a_last + 1 ? 0x07060302u : 0x05040100u, 0x07060302u};
    f32x4_t acc[MT][8];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[m][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int u) __attribute__((always_inline)) {
        u32x4_t fa[MT];
        if constexpr (DW) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
                fa[m] = u32x4_t{perm(af[u][1], af[u][0], a_sel[m]), perm(af[u][3], af[u][2], a_sel[m]),
                                perm(af[u][5], af[u][4], a_sel[m]), perm(af[u][7], af[u][6], a_sel[m])};
        } else {
#pragma unroll
            for (int m = 0; m < MT; ++m) fa[m] = u32x4_t{af[u][4 * m], af[u][4 * m + 1], af[u][4 * m + 2], af[u][4 * m + 3]};
        }
        float s2[2], s[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) s2[i] = DW ? mx_scale(sc[u][i]) : mx4_scale(sc[u][i]);
        static_for<0, 4>([&](auto q_c) __attribute__((always_inline)) {
            constexpr int Q = decltype(q_c)::value;
#pragma unroll
            for (int i = 0; i < 2; ++i) s[2 * Q + i] = __builtin_bit_cast(float, dpp_quad<0x55 * Q>(__builtin_bit_cast(uint32_t, s2[i])));
        });
        static_for<0, 4>([&](auto p_c) __attribute__((always_inline)) {
            constexpr int P = decltype(p_c)::value;                 // columns 2 P and 2 P + 1 of the lane's
            u32x4_t even, odd;
            if constexpr (DW) {
                // Products of codes and scales are bf16 numbers: their upper halves are all of them.
                uint32_t v[8][2];
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        v[i][h] = __builtin_bit_cast(uint32_t, float(int8_t(w[u][i][P / 2] >> (16 * (P & 1) + 8 * h))) * s[i]);
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    even[d] = perm(v[2 * d + 1][0], v[2 * d][0], 0x07060302u);
                    odd[d] = perm(v[2 * d + 1][1], v[2 * d][1], 0x07060302u);
                }
            } else {
                uint32_t v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u][i][0], s[i], P));
                even = pairs(v, 0);
                odd = pairs(v, 1);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                acc[m][2 * P] = mfma16_bf16(even, fa[m], acc[m][2 * P]);
                acc[m][2 * P + 1] = mfma16_bf16(odd, fa[m], acc[m][2 * P + 1]);
            }
        });
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n) load(u, u);
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
    if (cut) {
        load_cut(n, int(k_end - (k0 + 32 * int64_t(n))));
        multiply(0);
    }

    // Sum over the waves, 16 rows at a time, in a fixed order.  Piece v = 2 r + h of lane l holds columns
    // 32 g + 8 r + 4 h + 0..3; thread t then has columns 4 (t % 32) .. of row t / 32.  The pieces of
    // a row are 1 KiB apart, so their places are exchanged within 256 bytes by v and g.
    f32x4_t *const part = reinterpret_cast<f32x4_t *>(lds);         // [KW][8][64]
    const bool separate = a.g.reduce_in_kernel == REDUCE_SEPARATE;
    constexpr uint32_t SLICE = 8192 * MT;                            // a slice's partial sums
    const int tile = tm * a.g.tiles_n + tn;
    const __amdgpu_buffer_rsrc_t parts = mx_parts(a.g, tile, SLICE);
    const int row = int(threadIdx.x) >> 5, c4 = int(threadIdx.x) & 31;
    const int from_v = c4 & 7, from_g = c4 >> 3;
    const int from = from_v * 64 + from_g * 16 + (row ^ (from_v | (from_g & 1) << 3));
    const int64_t col = n0 + 4 * c4;
    auto row_of = [&](int m) __attribute__((always_inline)) { return DW ? m0 + 2 * row + m : m0 + 16 * m + row; };
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (m0 + (DW ? m : 16 * m) >= M) break;
        if (m > 0) __syncthreads();
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const int r = v >> 1, h = 4 * (v & 1);
            part[wave * 512 + v * 64 + grp * 16 + (l16 ^ (v | (grp & 1) << 3))] =
                f32x4_t{acc[m][h][r], acc[m][h + 1][r], acc[m][h + 2][r], acc[m][h + 3][r]};
        }
        __syncthreads();
        const int64_t at_m = row_of(m);
        if (at_m >= M || col >= N) continue;
        f32x4_t sum = part[from];
#pragma unroll
        for (int k = 1; k < KW; ++k) sum += part[k * 512 + from];
        if (a.g.split_k == 1) {
            mx_store4(a.g, at_m, col, sum);
        } else if (separate) {
            float *const plane = static_cast<float *>(a.g.workspace) + (slice * M + at_m) * N + col;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (col + r < N) plane[r] = sum[r];
        } else {
            mx_store_part(parts, slice * SLICE + m * 8192 + threadIdx.x * 16, sum);
        }
    }
    if (a.g.split_k == 1 || separate) return;
    if (!mx_last_slice(a.g, tile, *reinterpret_cast<int *>(lds))) return;
    f32x4_t total[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) total[m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int q = 0; q < a.g.split_k; q += 4) {           // four slices on the way; past the last one zeros
        f32x4_t v[4][MT];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m)
                v[u][m] = mx_load_part(parts, row_of(m) < M ? (q + u) * SLICE + m * 8192 + threadIdx.x * 16 : kOOB);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m) total[m] += v[u][m];
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
        if (row_of(m) < M && col < N) mx_store4(a.g, row_of(m), col, total[m]);
    mx_reset_counter(a.g, tile);
}

}  // namespace gemm
