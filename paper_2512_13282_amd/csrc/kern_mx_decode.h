// kern_mx_decode.h -- C = A . W^T for few rows of A: a read of the 4-bit weight.
#pragma once

#include "mx_common.h"

namespace gemm {

__device__ __forceinline__ f32x4_t mfma16_bf16(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                   0, 0, 0);
}

// Four consecutive results of row m from column col on, those past N left out.
__device__ __forceinline__ void mx_store4(const KernelArgs &g, int64_t m, int64_t col, f32x4_t v) {
    const int64_t at = m * g.ldc + col;
    if (g.epilogue == EPI_BF16) {
        uint16_t *const dst = static_cast<uint16_t *>(g.C) + at;
        const uint16_t o[4] = {bf16_nearest_even(v[0]), bf16_nearest_even(v[1]), bf16_nearest_even(v[2]), bf16_nearest_even(v[3])};
        if (col + 4 <= g.N) {
            store4<false>(dst, o);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (col + r < g.N) dst[r] = o[r];
        }
    } else {
        float *const dst = static_cast<float *>(g.C) + at;
        const float o[4] = {v[0], v[1], v[2], v[3]};
        if (col + 4 <= g.N) {
            store4<false>(dst, o);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (col + r < g.N) dst[r] = o[r];
        }
    }
}

// ---------------------------------------------------------------------------
// A workgroup holds 16 NT rows of W (columns of C), one of S slices of K and all rows of A, at
// most 16.  Its KW waves take contiguous parts of the slice and add their sums up in LDS.
//
// W goes straight from memory into registers, U chunks of 128 k on the way per wave: lane l
// loads the 16 bytes (one block of 32 codes) of row l % 16, block l / 16 of the chunk.  One
// conversion instruction turns two codes and the block's scale to bf16, and dword t of the
// sixteen bytes is the lane's share of the chunk's t-th 16 x 16 x 32 MFMA: lanes of group
// g = l / 16 hold k = 32 g + 8 t + 0..7, for W and for A.  The MFMAs multiply up to sixteen
// rows of A at the price of one; the matrix unit is idle otherwise, and the vector unit has
// the conversions to do.  Output register r of lane l is C[l % 16][4 (l / 16) + r].
//
// A's slice sits in LDS (rows 16 bytes past a multiple of 256, which puts sixteen rows on all
// banks; past the end of K zeros).
// ---------------------------------------------------------------------------
template <int NT, int KW, int U>
__global__ __launch_bounds__(64 * KW) void mx_decode_kernel(MxArgs a) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int l16 = lane & 15, grp = lane >> 4;
    const int64_t M = a.g.M, N = a.g.N, K = a.g.K;
    const int64_t n0 = int64_t(blockIdx.x) * (16 * NT);
    const int slice = int(blockIdx.y);

    // This workgroup's chunks, and this wave's.
    const int64_t chunks = (K + 127) / 128, whole = K / 128;
    const int64_t wg0 = slice * (a.g.k_chunk / 128);
    const int64_t wg1 = wg0 + a.g.k_chunk / 128 < chunks ? wg0 + a.g.k_chunk / 128 : chunks;
    const int per = int((wg1 - wg0 + KW - 1) / KW);
    const int64_t c0 = wg0 + wave * per;
    const int64_t end = c0 + per < wg1 ? c0 + per : wg1;
    const int n = int((end < whole ? end : whole) - c0);         // whole chunks; <= 0 for a wave without any

    // Rows past the end read the last one; their results are not stored.
    const uint8_t *wp[NT], *sp[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int64_t r = n0 + 16 * j + l16 < N ? n0 + 16 * j + l16 : N - 1;
        wp[j] = static_cast<const uint8_t *>(a.g.B) + r * a.g.ldb + c0 * 64 + 16 * grp;
        sp[j] = a.scales + r * a.ld_scales + c0 * 4;
    }
    u32x4_t w[U][NT];
    uint32_t sc[U][NT];
    auto load = [&](int u, int c) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            w[u][j] = *reinterpret_cast<const u32x4_any_mx *>(wp[j] + c * 64);
            sc[u][j] = *reinterpret_cast<const u32_any_mx *>(sp[j] + c * 4);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n) load(u, u);

    // A's slice into LDS.
    const int cols = int(wg1 - wg0) * 128, pitch = cols * 2 + 16;
    {
        const int pieces = cols / 8;                              // 16-byte pieces of a row
        const int64_t k0 = wg0 * 128;
        for (int p = int(threadIdx.x); p < int(M) * pieces; p += 64 * KW) {
            const int m = p / pieces, c = p - m * pieces;
            const uint16_t *const src = static_cast<const uint16_t *>(a.g.A) + m * a.g.lda + k0 + 8 * c;
            const int64_t left = K - k0 - 8 * c;
            u32x4_t v{0u, 0u, 0u, 0u};
            if (left >= 8) {
                v = *reinterpret_cast<const u32x4_any_mx *>(src);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < left) v[e / 2] |= uint32_t(src[e]) << (16 * (e & 1));
            }
            *reinterpret_cast<u32x4_t *>(lds + m * pitch + 16 * c) = v;
        }
    }
    __syncthreads();

    const uint8_t *const xrow = lds + (l16 < M ? l16 : int(M) - 1) * pitch + 64 * grp + int(c0 - wg0) * 256;
    f32x4_t acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](int u, int c) __attribute__((always_inline)) {
        u32x4_t x[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = *reinterpret_cast<const u32x4_t *>(xrow + c * 256 + 16 * t);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const float s = mx4_scale((sc[u][j] >> (8 * grp)) & 0xffu);
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[j] = mfma16_bf16(mx4_to_bf16(w[u][j][t], s), x[t], acc[j]);
        }
    };
    int i = 0;
    for (; i + 2 * U <= n; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            multiply(u, i + u);
            load(u, i + U + u);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (i + u < n) multiply(u, i + u);
        if (i + U + u < n) load(u, i + U + u);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (i + U + u < n) multiply(u, i + U + u);

    // The end of K that is no whole chunk, by the wave whose part it ends: dwords of eight
    // codes, and bytes within the last one.  Codes past the end meet A's zeros, under a
    // scale that is no NaN.
    if (chunks > whole && whole >= c0 && whole < end) {
        const int c = int(whole - c0);
        const int left = int(K - whole * 128) - 32 * grp;      // elements from this lane's block on
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            sc[0][j] = left > 0 ? uint32_t(sp[j][c * 4 + grp]) << (8 * grp) : 0u;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint8_t *const p = wp[j] + c * 64 + 4 * t;
                uint32_t v = 0;
                if (left >= 8 * (t + 1)) {
                    v = *reinterpret_cast<const u32_any_mx *>(p);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (8 * t + 2 * e < left) v |= uint32_t(p[e]) << (8 * e);
                }
                w[0][j][t] = v;
            }
        }
        multiply(0, c);
    }

    // Sum over the waves, in LDS (A is done with), in a fixed order.
    __syncthreads();
    f32x4_t *const part = reinterpret_cast<f32x4_t *>(lds);      // [KW][NT][64]
#pragma unroll
    for (int j = 0; j < NT; ++j) part[(wave * NT + j) * 64 + lane] = acc[j];
    __syncthreads();
    const bool separate = a.g.reduce_in_kernel == REDUCE_SEPARATE;
    const uint32_t bytes = NT * 1024;                            // a slice's partial sums
    const __amdgpu_buffer_rsrc_t parts = mx_parts(a.g, int(blockIdx.x), bytes);
    for (int s = int(threadIdx.x); s < NT * 64; s += 64 * KW) {
        const int64_t m = s & 15, col = n0 + 16 * (s >> 6) + 4 * ((s & 63) >> 4);
        if (m >= M || col >= N) continue;
        f32x4_t sum = part[s];
#pragma unroll
        for (int k = 1; k < KW; ++k) sum += part[k * NT * 64 + s];
        if (a.g.split_k == 1) {
            mx_store4(a.g, m, col, sum);
        } else if (separate) {
            float *const plane = static_cast<float *>(a.g.workspace) + (slice * M + m) * N + col;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (col + r < N) plane[r] = sum[r];
        } else {
            mx_store_part(parts, slice * bytes + s * 16, sum);
        }
    }
    if (a.g.split_k == 1 || separate) return;
    if (!mx_last_slice(a.g, int(blockIdx.x), *reinterpret_cast<int *>(lds + KW * NT * 1024))) return;
    for (int s = int(threadIdx.x); s < NT * 64; s += 64 * KW) {
        const int64_t m = s & 15, col = n0 + 16 * (s >> 6) + 4 * ((s & 63) >> 4);
        if (m >= M || col >= N) continue;
        f32x4_t sum{0.0f, 0.0f, 0.0f, 0.0f};
        for (int q = 0; q < a.g.split_k; q += 8) {       // eight loads on the way; past the last slice zeros
            f32x4_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = mx_load_part(parts, (q + u) * bytes + s * 16);
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u];
        }
        mx_store4(a.g, m, col, sum);
    }
    mx_reset_counter(a.g, int(blockIdx.x));
}

}  // namespace gemm
