// kern_adapters.h -- the adapters' first product and their weight gradients.
#pragma once

#include "adapters.h"
#include "fused_expand.h"
#include "kern_mx_decode.h"

namespace gemm {

// ---------------------------------------------------------------------------
// h of 16 MT tokens and 16 RT ranks over a slice of L, KW waves with a part of the slice each (16 x 16 x 32 MFMAs, Q the
// first operand: output register e of lane l is rank 4 (l / 16) + e of token l % 16).  Every element is used by
// one wave alone, so P, and Q where its rows lie along L, go from memory to registers, U chunks of 32 on the way; a Q
// that lies across passes through LDS of the wave's own and is read back transposed.  The adapters that occur among the
// tokens are taken one after the other over all rows, of which the adapter's own are written; the others' results are
// dropped.  `parts` workgroups share the adapters of the same tokens, in turn.
//
// Slices leave planes, which whoever reads h adds up.  Where `counters` is set they leave their sums as their registers
// hold them (a run of 1 KiB per wave and store), and the one that arrives last adds them up in their order (mx_common.h says
// how the accesses are ordered).
//
// Measured: 2048 x 4096 at rank 64 20.6 us, of which a floor of 4 is the read of x (element by element into h's shape the
// slices' sums took 5 us more); 16 x 14336 at rank 16, an adapter a token, 8.6: launch, index, two trips to memory, the sum.
// ---------------------------------------------------------------------------
template <bool QT, int MT, int RT, int KW>
__global__ __launch_bounds__(64 * KW) void adapters_shrink_kernel(ShrinkArgs s) {
    constexpr int PITCH = 32 * RT, CPR = 2 * RT;                 // bytes and 16-byte pieces of a row of Q across L
    __shared__ __attribute__((aligned(1024))) f32x4_t part[KW][MT * RT][64];
    static_assert(sizeof(part[0]) >= 32 * PITCH, "a wave's chunk of Q and its sums take turns");
    __shared__ int flag;
    const int lane = int(threadIdx.x) & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    const int l16 = lane & 15, grp = lane >> 4;
    const int block = int(blockIdx.x) / s.parts;
    const int64_t t0 = int64_t(block) * (16 * MT);
    int turn = int(blockIdx.x) % s.parts;                        // adapters until this workgroup's next
    const bool zeros = turn == 0;
    const int j0 = int(blockIdx.z) * (16 * RT);
    float *const out = s.out + int64_t(blockIdx.y) * s.plane;

    const int64_t l_begin = int64_t(blockIdx.y) * s.chunk, l_end = l_begin + s.chunk < s.L ? l_begin + s.chunk : s.L;
    const int length = int(l_end - l_begin), chunks = (length + 31) / 32, whole = length / 32, per = (chunks + KW - 1) / KW;
    const int c0 = wave * per, c1 = c0 + per < chunks ? c0 + per : chunks;
    const int n = (c1 < whole ? c1 : whole) - c0;                // whole chunks; <= 0 for a wave without any

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
        row[m] = static_cast<const uint16_t *>(s.P) + safe * s.ldp + l_begin + 32 * c0 + 8 * grp;
    }
    constexpr uint32_t TILES = MT * RT, SLICE = TILES * 1024;
    const int area = block * int(gridDim.z) + int(blockIdx.z);
    const __amdgpu_buffer_rsrc_t sums = make_rsrc(reinterpret_cast<uint8_t *>(s.out) + int64_t(area) * s.slices * SLICE, uint32_t(s.slices) * SLICE);
    auto to_h = [&](float *dst, int j, f32x4_t v) __attribute__((always_inline)) {
        if (j + 4 <= s.r) {
            *reinterpret_cast<f32x4_el_t *>(dst) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < s.r) dst[e] = v[e];
        }
    };
    // Tile k = RT m + rt: four ranks from j on of token t.
    auto store = [&](int k, int64_t t, f32x4_t v) __attribute__((always_inline)) {
        const int j = j0 + 16 * (k % RT) + 4 * grp;
        if (s.counters != nullptr) mx_store_part(sums, uint32_t(blockIdx.y) * SLICE + uint32_t(k * 1024 + lane * 16), v);
        else to_h(out + t * s.r + j, j, v);
    };
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int64_t t = t0 + 16 * m + l16;
        if (zeros && t < s.M && !has[m] && wave == m % KW)       // none: zeros
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) store(m * RT + rt, t, f32x4_t{0.0f, 0.0f, 0.0f, 0.0f});
    }
    for (;;) {
        int cur = -1;
#pragma unroll
        for (int m = MT - 1; m >= 0; --m)
            if (pending[m] != 0u) cur = __builtin_amdgcn_readlane(own[m], __builtin_ctz(pending[m]));
        if (cur < 0) break;
#pragma unroll
        for (int m = 0; m < MT; ++m) pending[m] &= ~uint32_t(__ballot(has[m] && own[m] == cur));
        if (turn-- > 0) continue;
        turn = s.parts - 1;
        const float scale = s.scale != nullptr ? s.scale[cur] : 1.0f;

        const uint16_t *const q = static_cast<const uint16_t *>(s.Q) + cur * s.sq;
        // Along L: rank l16 of tile rt.  Across: piece (lane % CPR) of row lane / CPR of each 64 / CPR rows.
        const uint16_t *qp[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if constexpr (QT) {
                const int j = j0 + 16 * rt + l16 < s.r ? j0 + 16 * rt + l16 : s.r - 1;      // past r: not written
                qp[rt] = q + j * s.ldq + l_begin + 32 * c0 + 8 * grp;
            } else {
                qp[rt] = q + (l_begin + 32 * c0 + rt * (64 / CPR) + lane / CPR) * s.ldq + j0 + 8 * (lane % CPR);
            }
        }
        const int ranks = s.r - j0 - 8 * (lane % CPR);           // of this lane's piece
        uint8_t *const mine = reinterpret_cast<uint8_t *>(part[wave]);

        f32x4_t acc[MT][RT];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[m][rt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        constexpr int U = MT * RT >= 8 ? 2 : MT * RT >= 4 ? 3 : 4;
        u32x4_t x[U][MT], w[U][RT];
        // Chunk c of this wave; rows of L past `left` are zeros.
        const bool pieces = s.r % 8 == 0;                        // Q across: whole pieces of ranks; those past r are not written
        if constexpr (!QT) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                if (pieces && ranks <= 0) qp[rt] -= 8 * (lane % CPR);
        }
        auto load = [&](int u, int c, bool all, bool eight) __attribute__((always_inline)) {
            const int left = length - 32 * (c0 + c);
#pragma unroll
            for (int m = 0; m < MT; ++m) x[u][m] = load8_bf16(row[m] + 32 * c, all ? 8 : left - 8 * grp);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if constexpr (QT) w[u][rt] = load8_bf16(qp[rt] + 32 * c, all ? 8 : left - 8 * grp);
                else w[u][rt] = load8_bf16(qp[rt] + 32 * c * s.ldq, all || rt * (64 / CPR) + lane / CPR < left ? (eight ? 8 : ranks) : 0);
            }
        };
        auto multiply = [&](int u) __attribute__((always_inline)) {
            u32x4_t f[RT];
            if constexpr (QT) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) f[rt] = w[u][rt];
            } else {
                auto swz_row = [](int r) { return RT == 4 ? ring_bswz<DT_BF16, 8>(r) : 0; };
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int r = rt * (64 / CPR) + lane / CPR;
                    *reinterpret_cast<u32x4_t *>(mine + r * PITCH + (((lane % CPR) ^ swz_row(r)) << 4)) = w[u][rt];
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // lanes read what others of the wave wrote
                const int r = 8 * grp + (l16 >> 2);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    const int colb = 32 * rt + 8 * (l16 & 3);
                    const uint8_t *const p = mine + r * PITCH + ((((colb >> 4) ^ swz_row(r)) << 4) | (colb & 15));
                    const u32x2_t lo = lds_read_tr<DT_BF16>(p), hi = lds_read_tr<DT_BF16>(p + 4 * PITCH);
                    f[rt] = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[m][rt] = mfma16_bf16(f[rt], x[u][m], acc[m][rt]);
        };
        auto walk = [&](auto eight_c) __attribute__((always_inline)) {
            constexpr bool EIGHT = decltype(eight_c)::value;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (u < n) load(u, u, true, EIGHT);
            int i = 0;
            for (; i + 2 * U <= n; i += U) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    multiply(u);
                    load(u, i + U + u, true, EIGHT);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u < n) multiply(u);
                if (i + U + u < n) load(u, i + U + u, true, EIGHT);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + U + u < n) multiply(u);
        };
        if (QT || pieces) walk(std::true_type{});
        else walk(std::false_type{});
        if (chunks > whole && whole >= c0 && whole < c1) {       // the end of L that is no whole chunk
            load(0, whole - c0, false, false);
            multiply(0);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) part[wave][m * RT + rt][lane] = acc[m][rt];
        phase_barrier();
        for (int k = wave; k < MT * RT; k += KW) {
            f32x4_t sum = part[0][k][lane];
#pragma unroll
            for (int v = 1; v < KW; ++v) sum += part[v][k][lane];
            const int m = k / RT;
            bool take = false;
#pragma unroll
            for (int v = 0; v < MT; ++v)
                if (v == m) take = has[v] && own[v] == cur;
            if (take) store(k, t0 + 16 * m + l16, sum * scale);
        }
        phase_barrier();
    }
    if (s.counters == nullptr) return;
    // The last of the block's slices and parts adds the planes up.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
        flag = __hip_atomic_fetch_add(&s.counters[area], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == unsigned(s.slices * s.parts - 1);
    __syncthreads();
    if (flag == 0) return;
    for (int k = wave; k < int(TILES); k += KW) {
        const int64_t t = t0 + 16 * (k / RT) + l16;
        f32x4_t v[8];                                            // past the last slice zeros
#pragma unroll
        for (int p = 0; p < 8; ++p) v[p] = mx_load_part(sums, t < s.M ? uint32_t(p) * SLICE + uint32_t(k * 1024 + lane * 16) : kOOB);
        f32x4_t sum = v[0];
#pragma unroll
        for (int p = 1; p < 8; ++p) sum += v[p];
        const int j = j0 + 16 * (k % RT) + 4 * grp;
        if (t < s.M) to_h(s.h + t * s.r + j, j, sum);
    }
    if (threadIdx.x == 0) __hip_atomic_store(&s.counters[area], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---------------------------------------------------------------------------
// One adapter's gradient over 64 columns of z (x for dA, dy for dB) and 16 RT ranks: T[c][j] = sum z[t][c] h[t][j] over
// the adapter's tokens.  Four waves scan the index 64 tokens at a time, in turn, and put the adapter's into a list of
// their own; 32 of them are a step of 16 x 16 x 32 MFMAs.  Rows of z pass through LDS and are read back
// transposed; h keeps its fp32 value in bf16 parts (split_bf16).  The waves' sums meet in LDS in a fixed order, so
// results do not depend on timing.  Rows of other adapters are never read.
//
// Measured: 2048 tokens of eight adapters of rank 16, x 4096 and dy 11008 wide, 22 to 24 us for 62 MB read (a look at the index at a
// time instead of eight 2 us more).  Registers are held to as many workgroups as LDS leaves room for on a compute unit, five at rank 16:
// with the second walk's they would be four.
// ---------------------------------------------------------------------------
template <int RT>
__global__ __launch_bounds__(256, RT == 1 ? 5 : RT == 2 ? 3 : 2) void adapters_dw_kernel(AdapterDwArgs a) {
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

    // A step over list entries [head, head + 32), the first `count` of them.
    int head = 0, held = 0;
    auto step = [&](int count, auto strict_c) __attribute__((always_inline)) {
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
                const u32x4_t finite = decltype(strict_c)::value ? finite_bf16(zf[c]) : zf[c];
                if (exact) acc[i][c] = mfma16_bf16(h3[2], finite, acc[i][c]);
                acc[i][c] = mfma16_bf16(h3[1], finite, acc[i][c]);
                acc[i][c] = mfma16_bf16(h3[0], zf[c], acc[i][c]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        head = (head + 32) & 127;
        held -= 32;
    };

    constexpr int LOOKS = 8;                                     // looks at the index on the way at once
    auto walk = [&](auto strict_c) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int c = 0; c < CT; ++c) acc[i][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        head = held = 0;
        for (int64_t t0 = int64_t(wave) * 64; t0 < a.M; t0 += 64 * WAVES * LOOKS) {
            int own[LOOKS];
#pragma unroll
            for (int k = 0; k < LOOKS; ++k) {
                const int64_t t = t0 + 64 * WAVES * k + lane;
                own[k] = t < a.M ? a.index[t] : -1;
            }
#pragma unroll 1
            for (int k = 0; k < LOOKS; ++k) {
                const uint64_t mask = __ballot(own[0] == cur);
                const int t = int(t0) + 64 * WAVES * k + lane;
                const bool mine = own[0] == cur;
#pragma unroll
                for (int i = 0; i + 1 < LOOKS; ++i) own[i] = own[i + 1];
                if (mask == 0u) continue;
                if (mine) {
                    const int before = __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0u));
                    list[wave][(head + held + before) & 127] = t;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                held += __builtin_popcountll(mask);                  // at most 31 + 64
                while (held >= 32) step(32, strict_c);
            }
        }
        if (held > 0) step(held, strict_c);
    };
    walk(std::false_type{});
    // Sums that are not all finite are formed again, from rows without their infinities and NaN where a part of h may not
    // meet them (finite_bf16).
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) all = __builtin_fmaf(acc[i][c][e], 0.0f, all);
    if (__ballot(all != all) != 0u) walk(std::true_type{});

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
