// kern_adapters.h -- the adapters' first product and their weight gradients.
#pragma once

#include "adapters.h"
#include "fused_expand.h"
#include "kern_mx_decode.h"

namespace gemm {

// Eight bf16 values at any address, the first `left` of them, zeros after them.
__device__ __forceinline__ u32x4_t load8_bf16(const uint16_t *p, int64_t left) {
    u32x4_t v{0u, 0u, 0u, 0u};
    if (left >= 8) {
        v = *reinterpret_cast<const u32x4_el2_t *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) v[e / 2] |= uint32_t(p[e]) << (16 * (e & 1));
    }
    return v;
}

// ---------------------------------------------------------------------------
// h of 16 MT tokens and 16 RT ranks over a slice of L, KW waves with a part of the slice each (16 x 16 x 32 MFMAs, Q the
// first operand: output register e of lane l is rank 4 (l / 16) + e of token l % 16).  Both operands go from memory to
// registers, for every element is used by one wave alone.  The adapters that occur among the tokens are taken one after
// the other over all rows, of which the adapter's own are written; the others' results are dropped.
// Slices leave planes that whoever reads h adds up in their order.
// ---------------------------------------------------------------------------
template <bool QT, int MT, int RT, int KW>
__global__ __launch_bounds__(64 * KW) void adapters_shrink_kernel(ShrinkArgs s) {
    __shared__ __attribute__((aligned(16))) f32x4_t part[KW][MT * RT][64];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    const int64_t t0 = int64_t(blockIdx.x) * (16 * MT);
    const int j0 = int(blockIdx.z) * (16 * RT);
    float *const out = s.out + int64_t(blockIdx.y) * s.plane;

    const int64_t l_begin = int64_t(blockIdx.y) * s.chunk, l_end = l_begin + s.chunk < s.L ? l_begin + s.chunk : s.L;
    const int chunks = int((l_end - l_begin + 31) / 32), per = (chunks + KW - 1) / KW;
    const int c0 = wave * per, c1 = c0 + per < chunks ? c0 + per : chunks;

    int own[MT];
    bool has[MT];
    uint32_t pending[MT];
    const uint16_t *row[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t t = t0 + 16 * m + l16, safe = t < s.M ? t : s.M - 1;
        own[m] = s.n > 0 ? s.index[safe] : -1;
        has[m] = t < s.M && uint32_t(own[m]) < uint32_t(s.n);
        pending[m] = uint32_t(__ballot(has[m])) & 0xffffu;
        row[m] = static_cast<const uint16_t *>(s.P) + safe * s.ldp + l_begin + 8 * grp;
        if (t < s.M && !has[m] && wave == m % KW) {              // none: zeros
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j0 + 16 * rt + 4 * grp + e < s.r) out[t * s.r + j0 + 16 * rt + 4 * grp + e] = 0.0f;
        }
    }
    for (;;) {
        int cur = -1;
#pragma unroll
        for (int m = MT - 1; m >= 0; --m)
            if (pending[m] != 0u) cur = __builtin_amdgcn_readlane(own[m], __builtin_ctz(pending[m]));
        if (cur < 0) break;
#pragma unroll
        for (int m = 0; m < MT; ++m) pending[m] &= ~uint32_t(__ballot(has[m] && own[m] == cur));

        const uint16_t *const q = static_cast<const uint16_t *>(s.Q) + cur * s.sq;
        const uint16_t *qp[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int j = j0 + 16 * rt + l16 < s.r ? j0 + 16 * rt + l16 : s.r - 1;      // past r: not written
            qp[rt] = QT ? q + j * s.ldq + l_begin + 8 * grp : q + (l_begin + 8 * grp) * s.ldq + j;
        }
        f32x4_t acc[MT][RT];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[m][rt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        auto load = [&](int c, u32x4_t (&x)[MT], u32x4_t (&w)[RT], int64_t left) __attribute__((always_inline)) {
#pragma unroll
            for (int m = 0; m < MT; ++m) x[m] = load8_bf16(row[m] + 32 * c, left);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if constexpr (QT) {
                    w[rt] = load8_bf16(qp[rt] + 32 * c, left);
                } else {
                    w[rt] = u32x4_t{0u, 0u, 0u, 0u};
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e < left) w[rt][e / 2] |= uint32_t(qp[rt][(32 * c + e) * s.ldq]) << (16 * (e & 1));
                }
            }
        };
        auto multiply = [&](const u32x4_t (&x)[MT], const u32x4_t (&w)[RT]) __attribute__((always_inline)) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[m][rt] = mfma16_bf16(w[rt], x[m], acc[m][rt]);
        };
        constexpr int U = RT >= 4 ? 2 : 4;                       // chunks on the way at once
        const int64_t mine = l_end - l_begin - 8 * grp;         // from this lane's first element on
        int c = c0;
        for (; c + U <= c1 && 32 * int64_t(c + U) <= l_end - l_begin; c += U) {
            u32x4_t x[U][MT], w[U][RT];
#pragma unroll
            for (int u = 0; u < U; ++u) load(c + u, x[u], w[u], 8);
#pragma unroll
            for (int u = 0; u < U; ++u) multiply(x[u], w[u]);
        }
        for (; c < c1; ++c) {
            u32x4_t x[MT], w[RT];
            load(c, x, w, mine - 32 * int64_t(c));
            multiply(x, w);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) part[wave][m * RT + rt][lane] = acc[m][rt];
        __syncthreads();
        const float scale = s.scale != nullptr ? s.scale[cur] : 1.0f;
        for (int i = wave; i < MT * RT; i += KW) {
            f32x4_t sum = part[0][i][lane];
#pragma unroll
            for (int k = 1; k < KW; ++k) sum += part[k][i][lane];
            const int m = i / RT, j = j0 + 16 * (i % RT) + 4 * grp;
            const int64_t t = t0 + 16 * m + l16;
            bool take = false;
#pragma unroll
            for (int v = 0; v < MT; ++v)
                if (v == m) take = has[v] && own[v] == cur;
            if (take) {
                float *const dst = out + t * s.r + j;
                if (j + 4 <= s.r) {
                    *reinterpret_cast<f32x4_el_t *>(dst) = sum * scale;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (j + e < s.r) dst[e] = sum[e] * scale;
                }
            }
        }
        __syncthreads();
    }
}

// h = the sum of its planes, where the caller keeps it.
__global__ __launch_bounds__(256) void adapters_sum_kernel(const float *__restrict__ parts, int64_t plane, int slices, float *__restrict__ h, int64_t total) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        float v = 0.0f;
        for (int p = 0; p < slices; ++p) v += parts[p * plane + i];
        h[i] = v;
    }
}

// ---------------------------------------------------------------------------
// One adapter's gradient over 64 columns of z (x for dA, dy for dB) and 16 RT ranks: T[c][j] = sum z[t][c] h[t][j] over
// the adapter's tokens.  Four waves scan the index 64 tokens at a time, in turn, and put the adapter's into a list of
// their own; 32 of them are a step of 16 x 16 x 32 MFMAs.  Rows of z pass through LDS and are read back
// transposed; h keeps its fp32 value in bf16 parts (split_bf16).  The waves' sums meet in LDS in a fixed order, so
// results do not depend on timing.  Rows of other adapters are never read.
// ---------------------------------------------------------------------------
template <int RT>
__global__ __launch_bounds__(256) void adapters_dw_kernel(AdapterDwArgs a) {
    constexpr int WAVES = 4, CT = 4;                             // column tiles of 16
    __shared__ __attribute__((aligned(1024))) uint8_t rows[WAVES][32 * 128];
    __shared__ int list[WAVES][128];
    __shared__ __attribute__((aligned(16))) f32x4_t part[WAVES - 1][RT * CT][64];
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    const bool second = int(blockIdx.x) >= a.side[0].blocks;
    const AdapterDwArgs::Side &side = a.side[second ? 1 : 0];
    const int64_t col0 = int64_t(int(blockIdx.x) - (second ? a.side[0].blocks : 0)) * 64;
    const int cur = int(blockIdx.y), j0 = int(blockIdx.z) * (16 * RT);
    const uint16_t *const z = static_cast<const uint16_t *>(side.z);
    const bool exact = !a.bf16_out;

    f32x4_t acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[i][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    // A step over list entries [head, head + 32), the first `count` of them.
    int head = 0, held = 0;
    auto step = [&](int count) __attribute__((always_inline)) {
        u32x4_t zv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {                            // lane: row 8 i + lane / 8, 16 bytes lane % 8
            const int r = 8 * i + (lane >> 3);
            const int t = list[wave][(head + r) & 127];
            const int64_t col = col0 + 8 * (lane & 7);
            zv[i] = load8_bf16(z + int64_t(r < count ? t : 0) * side.ldz + col, r < count ? side.cols - col : 0);
        }
        float hv[RT][8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {                            // lane: tokens 8 grp + e, rank l16 of each tile
            const int r = 8 * grp + e;
            const int t = list[wave][(head + r) & 127];
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int j = j0 + 16 * i + l16;
                hv[i][e] = r < count && j < a.r ? side.h[int64_t(t) * a.r + j] : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 8 * i + (lane >> 3);
            *reinterpret_cast<u32x4_t *>(rows[wave] + r * 128 + (((lane & 7) ^ ring_bswz<DT_BF16, 8>(r)) << 4)) = zv[i];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // lanes read what others of the wave wrote
        // Transpose reads: lane g of a group of 16 addresses row g / 4, columns 4 (g % 4) .. + 3, and receives column g.
        u32x4_t zf[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int r = 8 * grp + (l16 >> 2), colb = 32 * c + 8 * (l16 & 3);
            const uint8_t *const p = rows[wave] + r * 128 + ((((colb >> 4) ^ ring_bswz<DT_BF16, 8>(r)) << 4) | (colb & 15));
            const u32x2_t lo = lds_read_tr<DT_BF16>(p), hi = lds_read_tr<DT_BF16>(p + 4 * 128);
            zf[c] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            u32x4_t h3[3];
            split_bf16(hv[i], h3);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                if (exact) acc[i][c] = mfma16_bf16(h3[2], zf[c], acc[i][c]);
                acc[i][c] = mfma16_bf16(h3[1], zf[c], acc[i][c]);
                acc[i][c] = mfma16_bf16(h3[0], zf[c], acc[i][c]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        head = (head + 32) & 127;
        held -= 32;
    };

    for (int64_t t0 = int64_t(wave) * 64; t0 < a.M; t0 += 64 * WAVES) {
        const int64_t t = t0 + lane;
        const bool mine = t < a.M && a.index[t] == cur;
        const uint64_t mask = __ballot(mine);
        if (mask == 0u) continue;
        if (mine) {
            const int before = __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0u));
            list[wave][(head + held + before) & 127] = int(t);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        held += __builtin_popcountll(mask);                      // at most 31 + 64
        while (held >= 32) step(32);
    }
    if (held > 0) step(held);

    // The waves' sums, wave 0's first.
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) part[wave - 1][i * CT + c][lane] = acc[i][c];
    }
    __syncthreads();
    if (wave > 0) return;
    // Register e of lane l: rank 4 (l / 16) + e, column l % 16.
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            f32x4_t sum = acc[i][c];
#pragma unroll
            for (int w = 0; w < WAVES - 1; ++w) sum += part[w][i * CT + c][lane];
            const int64_t col = col0 + 16 * c + l16;
            const int j = j0 + 16 * i + 4 * grp;
            if (col >= side.cols) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (j + e >= a.r) continue;
                const int64_t at = cur * side.stride + (second ? col * side.ld + j + e : (j + e) * side.ld + col);
                if (a.bf16_out) static_cast<uint16_t *>(side.out)[at] = bf16_nearest_even(sum[e]);
                else static_cast<float *>(side.out)[at] = sum[e];
            }
        }
}

}  // namespace gemm
