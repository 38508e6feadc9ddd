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
// A workgroup holds 16 rows of W (columns of C), one of S slices of K and all rows of A, at
// most 16 MT.  Its KW waves take contiguous parts of the slice and add their sums up in LDS.
// Neither operand has to lie on aligned rows.
//
// W goes straight from memory into registers, U chunks of 128 k on the way per wave: lane l
// loads the 16 bytes (one block of 32 codes) of row l % 16, block l / 16 of the chunk.  One
// conversion instruction turns two codes and the block's scale to bf16, and dword t of the
// sixteen bytes is the lane's share of the chunk's t-th 16 x 16 x 32 MFMA: lanes of group
// g = l / 16 hold k = 32 g + 8 t + 0..7, for W and for A.  The MFMAs multiply up to sixteen
// rows of A at the price of one; the matrix unit is idle otherwise, and the vector unit has
// the conversions to do.  Output register r of lane l is C[l % 16][4 (l / 16) + r].  MT = 3 serves
// 17 to 48 rows whose operands the tile kernels would have copied first (37 x 2051 x 2049: a launch
// and 3 us less).
//
// A's slice sits in LDS (rows 16 bytes past a multiple of 256, which puts sixteen rows on all
// banks; past the end of K zeros).  Its first pieces are loaded ahead of W's, so that writing them
// does not wait for memory: loads complete in order.
//
// Bound by the read of W.  1 x 14336 x 4096 (31 MB): 9.7 us, of which an empty launch is 2.5;
// 1 x 4096 x 14336: 8.5; 1 x 11008 x 4096: 8.1.  Measured against it: A read per lane from memory
// 9.6 to 9.9 at 1 x 4096 x 14336 (its fragments take the load path four times W's); A after W 9.0;
// 32 rows of W to a workgroup 10 and more; four waves with four chunks each 9.4 at 1 x 14336 x 4096,
// but 8.2 at 1 x 11008 x 4096 and 11.0 against 10.1 at 2 x 14336 x 4096; non-temporal loads of W 9.9.
// ---------------------------------------------------------------------------
template <int MT, int KW, int U>
__global__ __launch_bounds__(64 * KW) void mx_decode_kernel(MxArgs a) {
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = int(threadIdx.x) & 63, wave = int(threadIdx.x) >> 6;
    const int l16 = lane & 15, grp = lane >> 4;
    const int64_t M = a.g.M, N = a.g.N, K = a.g.K;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const int slice = int(blockIdx.y);

    // This workgroup's chunks, and this wave's.
    const int64_t chunks = (K + 127) / 128, whole = K / 128;
    const int64_t wg0 = slice * (a.g.k_chunk / 128);
    const int64_t wg1 = wg0 + a.g.k_chunk / 128 < chunks ? wg0 + a.g.k_chunk / 128 : chunks;
    const int per = int((wg1 - wg0 + KW - 1) / KW);
    const int64_t c0 = wg0 + wave * per;
    const int64_t end = c0 + per < wg1 ? c0 + per : wg1;
    const int n = int((end < whole ? end : whole) - c0);         // whole chunks; <= 0 for a wave without any

    // Piece p of A's slice: 16 bytes of a row.
    const int cols = int(wg1 - wg0) * 128, pitch = cols * 2 + 16, pieces = cols / 8, total = int(M) * pieces;
    const int64_t k0 = wg0 * 128;
    auto fetch = [&](int p) __attribute__((always_inline)) {
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
        return v;
    };
    auto put = [&](int p, u32x4_t v) __attribute__((always_inline)) {
        const int m = p / pieces, c = p - m * pieces;
        *reinterpret_cast<u32x4_t *>(lds + m * pitch + 16 * c) = v;
    };
    u32x4_t first{0u, 0u, 0u, 0u};
    if (int(threadIdx.x) < total) first = fetch(int(threadIdx.x));

    // A row past the end reads the last one; its results are not stored.
    const int64_t row = n0 + l16 < N ? n0 + l16 : N - 1;
    const uint8_t *const wp = static_cast<const uint8_t *>(a.g.B) + row * a.g.ldb + c0 * 64 + 16 * grp;
    const uint8_t *const sp = a.scales + row * a.ld_scales + c0 * 4;
    u32x4_t w[U];
    uint32_t sc[U];
    auto load = [&](int u, int c) __attribute__((always_inline)) {
        w[u] = *reinterpret_cast<const u32x4_any_mx *>(wp + c * 64);
        sc[u] = *reinterpret_cast<const u32_any_mx *>(sp + c * 4);
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n) load(u, u);

    if (int(threadIdx.x) < total) put(int(threadIdx.x), first);
    for (int p = int(threadIdx.x) + 64 * KW; p < total; p += 64 * KW) put(p, fetch(p));
    __syncthreads();

    const uint8_t *xrow[MT];
    f32x4_t acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        xrow[m] = lds + (16 * m + l16 < M ? 16 * m + l16 : int(M) - 1) * pitch + 64 * grp + int(c0 - wg0) * 256;
        acc[m] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
    auto multiply = [&](int u, int c) __attribute__((always_inline)) {
        const float s = mx4_scale((sc[u] >> (8 * grp)) & 0xffu);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const u32x4_t wf = mx4_to_bf16(w[u][t], s);
#pragma unroll
            for (int m = 0; m < MT; ++m)
                acc[m] = mfma16_bf16(wf, *reinterpret_cast<const u32x4_t *>(xrow[m] + c * 256 + 16 * t), acc[m]);
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
    // codes, and bytes within the last one.  Past the end codes are zeros under a scale that is
    // no NaN, the unused half of an odd row's last byte too: it may stand for an infinity.
    if (chunks > whole && whole >= c0 && whole < end) {
        const int c = int(whole - c0);
        const int left = int(K - whole * 128) - 32 * grp;      // elements from this lane's block on
        sc[0] = left > 0 ? uint32_t(sp[c * 4 + grp]) << (8 * grp) : 0u;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint8_t *const p = wp + c * 64 + 4 * t;
            uint32_t v = 0;
            if (left >= 8 * (t + 1)) {
                v = *reinterpret_cast<const u32_any_mx *>(p);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (8 * t + 2 * e < left) v |= uint32_t(p[e]) << (8 * e);
            }
            w[0][t] = v;
        }
        w[0] = mx4_first(w[0], left);
        multiply(0, c);
    }

    // Sum over the waves, in LDS (A is done with), in a fixed order.
    __syncthreads();
    f32x4_t *const part = reinterpret_cast<f32x4_t *>(lds);      // [KW][MT][64]
#pragma unroll
    for (int m = 0; m < MT; ++m) part[(wave * MT + m) * 64 + lane] = acc[m];
    __syncthreads();
    const bool separate = a.g.reduce_in_kernel == REDUCE_SEPARATE;
    constexpr uint32_t BYTES = 1024 * MT;                        // a slice's partial sums
    const __amdgpu_buffer_rsrc_t parts = mx_parts(a.g, int(blockIdx.x), BYTES);
    const int64_t m = 16 * wave + l16, col = n0 + 4 * grp;       // wave w < MT has rows 16 w ..
    const bool holds = wave < MT && m < M && col < N;
    const uint32_t at = uint32_t(wave * 64 + lane);
    if (holds) {
        f32x4_t sum = part[at];
#pragma unroll
        for (int k = 1; k < KW; ++k) sum += part[k * MT * 64 + at];
        if (a.g.split_k == 1) {
            mx_store4(a.g, m, col, sum);
        } else if (separate) {
            float *const plane = static_cast<float *>(a.g.workspace) + (slice * M + m) * N + col;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (col + r < N) plane[r] = sum[r];
        } else {
            mx_store_part(parts, slice * BYTES + at * 16, sum);
        }
    }
    if (a.g.split_k == 1 || separate) return;
    if (!mx_last_slice(a.g, int(blockIdx.x), *reinterpret_cast<int *>(lds + KW * MT * 1024))) return;
    if (holds) {
        f32x4_t sum{0.0f, 0.0f, 0.0f, 0.0f};
        for (int q = 0; q < a.g.split_k; q += 8) {       // eight loads on the way; past the last slice zeros
            f32x4_t v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = mx_load_part(parts, (q + u) * BYTES + at * 16);
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u];
        }
        mx_store4(a.g, m, col, sum);
    }
    mx_reset_counter(a.g, int(blockIdx.x));
}

}  // namespace gemm
