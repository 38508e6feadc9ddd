// fused_expand.h -- the adapters' second product, h Q_i, onto a wave's sums.
#pragma once

#include "fused_common.h"

namespace gemm {

typedef float f32x4_el_t __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x4_el2_t __attribute__((ext_vector_type(4), aligned(2)));

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

// Eight floats as bf16 parts whose sum they are: the upper 8 bits of each, what is left rounded to 8 bits, and what that leaves
// (24 bits in all, so three parts are exact; two leave half a step of the second, 2^-16).  An infinity or a NaN is its own
// first part.
__device__ __forceinline__ void split_bf16(const float (&v)[8], u32x4_t (&part)[3]) {
    uint32_t b[8];
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t x = __builtin_bit_cast(uint32_t, v[e]);
        const bool finite = (x & 0x7f800000u) != 0x7f800000u;
        b[e] = finite || (x & 0x007fffffu) == 0u ? x : x | 0x00400000u;
        rest[e] = finite ? v[e] - __builtin_bit_cast(float, x & 0xffff0000u) : 0.0f;
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const uint32_t second = pack_bf16(rest[2 * d], rest[2 * d + 1]);
        part[0][d] = perm(b[2 * d + 1], b[2 * d], 0x07060302u);
        part[1][d] = second;
        part[2][d] = pack_bf16(rest[2 * d] - bf16_to_f32(second & 0xffffu), rest[2 * d + 1] - bf16_to_f32(second >> 16));
    }
}

// The finite ones of eight bf16 values, zeros in the others' places.  Where a factor in parts meets an infinity, its second
// and third part, 0 or of the other sign, would make a NaN of what the factor itself only gives its sign: they take these, and the
// first part, the factor's upper bits, takes the values as they are.
__device__ __forceinline__ u32x4_t finite_bf16(u32x4_t w) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const uint32_t t = ((w[d] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;      // an exponent of all ones
        w[d] &= ~((t << 1) - (t >> 15));
    }
    return w;
}

// Row t's h from element k on, the first `left` of eight, summed over its planes in their order.
__device__ __forceinline__ void load_h(const FusedArgs &a, int64_t t, int k, int left, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    for (int p = 0; p < a.planes; ++p) {                         // one, but for few rows
        const float *const src = a.h + p * a.h_plane + t * a.r + k;
        if (left >= 8) {
            const f32x4_t x = *reinterpret_cast<const f32x4_el_t *>(src), y = *reinterpret_cast<const f32x4_el_t *>(src + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] += x[e];
                v[4 + e] += y[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left) v[e] += src[e];
        }
    }
}

// Eight bf16 values at any address, all of them inside the matrix.  ODD: the address may be off a dword, where a
// 16-byte load takes 2.4 times as long (gated 37 x 2048 x 2049 against x 2050: 23.3 and 9.8 us): dwords from the
// one that holds the first value, and one more, put together.
template <bool ODD>
__device__ __forceinline__ u32x4_t load8_any(const uint16_t *p) {
    if constexpr (!ODD) {
        return *reinterpret_cast<const u32x4_el2_t *>(p);
    } else {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        const uint32_t *const q = reinterpret_cast<const uint32_t *>(at & ~uintptr_t(3));
        const uint32_t shift = uint32_t(at & 2) * 8;
        const u32x4_t v = *reinterpret_cast<const u32x4_el_t *>(q);
        const uint32_t last = q[shift ? 4 : 3];
        return u32x4_t{__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift),
                       __builtin_amdgcn_alignbit(v[3], v[2], shift), __builtin_amdgcn_alignbit(last, v[3], shift)};
    }
}

// ---------------------------------------------------------------------------
// acc += h_t Q_i(t) for the wave's rows (TM x 32 from r0) and columns (32 from c0 and 32 from c0 + HALF).  QT: Q_i
// is N x r, else r x N.
//
// Rows of one adapter take its product straight onto their sums.  Among others the adapters that occur in 32 rows are
// taken one after the other (a decode batch's rows of weights have to be read for each of its requests anyway), each as
// a product of the 32 rows, of which only the adapter's own take the result: rows are chosen, not multiplied
// by zeros, so an infinity or a NaN in one request's adapter stays out of the others'.  h does not depend on the
// adapter and is read once for every 16 ranks; the matrices of two to four adapters are on their way at once, for what
// a batch of many requests waits for is their latency.  h keeps its fp32 value in two bf16 parts (2^-16 left
// out, a bf16 result's half step being 2^-8), three and so all of it for an fp32 result.  Runs ahead of the
// K loop, on sums that are 0, while the first stages are on their way.
//
// Sums that are not all finite are formed again, STRICT, from values without their infinities and NaN where a part of h may not
// meet them (finite_bf16).  One look at the sums costs products of finite values next to nothing; values taken out of every product cost
// the gradients of adapters.h (4096 and 11008 wide, 2048 tokens, rank 16) 22.5 -> 26 us, 2048 tokens in no order at rank 64 223 -> 240.
// ---------------------------------------------------------------------------
template <bool QT, int HALF, bool STRICT, int TM, int TN>
__device__ __forceinline__ void expand_adapters_as(const FusedArgs &a, f32x16_t (&acc)[TM][TN], int64_t r0, int64_t c0, int lane) {
    const int l32 = lane & 31, half = lane >> 5;
    const bool exact = a.g.epilogue != EPI_BF16;
    const int64_t N = a.g.N;
    int64_t col[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t c = c0 + HALF * j + l32;
        col[j] = c < N ? c : N - 1;                              // not stored
    }
    // Eight of column c's values from rank k0 on.
    auto weights = [&](const uint16_t *q, int64_t c, int k0, int left) __attribute__((always_inline)) {
        if (QT) return load8_bf16(q + c * a.ldq + k0, left);
        u32x4_t w{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) w[e / 2] |= uint32_t(q[(k0 + e) * a.ldq + c]) << (16 * (e & 1));
        return w;
    };
    int own[TM];
    uint32_t all[TM];
    int common = -1;                                             // the adapter of all rows, if it is one
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t t = r0 + 32 * i + l32;
        own[i] = t < a.g.M ? a.index[t] : -1;
        if (uint32_t(own[i]) >= uint32_t(a.n)) own[i] = -1;
        all[i] = uint32_t(__ballot(own[i] >= 0));
        if (all[i] != 0u && common < 0) common = __builtin_amdgcn_readlane(own[i], __builtin_ctz(all[i]));
    }
    if (common < 0) return;
    uint32_t others = 0u;
#pragma unroll
    for (int i = 0; i < TM; ++i) others |= uint32_t(__ballot(r0 + 32 * i + l32 < a.g.M && own[i] != common));
    if (others == 0u) {
        // One for all rows: straight onto the sums, its matrix read once.
        const uint16_t *const q = static_cast<const uint16_t *>(a.Q) + common * a.sq;
        for (int k = 0; k < a.r; k += 16) {
            const int k0 = k + 8 * half, left = a.r - k0;
            u32x4_t w[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) w[j] = weights(q, col[j], k0, left);
            float v[TM][8] = {};
#pragma unroll
            for (int i = 0; i < TM; ++i)
                if (own[i] >= 0) load_h(a, r0 + 32 * i + l32, k0, left, v[i]);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                u32x4_t part[3];
                split_bf16(v[i], part);
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const u32x4_t finite = STRICT ? finite_bf16(w[j]) : w[j];
                    if (exact) acc[i][j] = mfma32<DT_BF16>(part[2], finite, acc[i][j]);
                    acc[i][j] = mfma32<DT_BF16>(part[1], finite, acc[i][j]);
                    acc[i][j] = mfma32<DT_BF16>(part[0], w[j], acc[i][j]);
                }
            }
        }
        return;
    }
    static_for<0, TM>([&](auto i_c) __attribute__((always_inline)) {
        constexpr int I = decltype(i_c)::value;
        if (all[I] == 0u) return;
        for (int k = 0; k < a.r; k += 16) {
            const int k0 = k + 8 * half, left = a.r - k0;
            float v[8] = {};
            if (own[I] >= 0) load_h(a, r0 + 32 * I + l32, k0, left, v);
            u32x4_t part[3];
            split_bf16(v, part);
            constexpr int B = TM > 3 ? 2 : 4;                    // adapters on the way at once
            uint32_t pending = all[I];
            while (pending != 0u) {
                u32x4_t w[B][TN];
                uint32_t rows[B];
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    rows[b] = 0u;
                    if (pending == 0u) continue;
                    const int cur = __builtin_amdgcn_readlane(own[I], __builtin_ctz(pending));
                    rows[b] = uint32_t(__ballot(own[I] == cur));
                    pending &= ~rows[b];
                    const uint16_t *const q = static_cast<const uint16_t *>(a.Q) + cur * a.sq;
#pragma unroll
                    for (int j = 0; j < TN; ++j) w[b][j] = weights(q, col[j], k0, left);
                }
#pragma unroll
                for (int b = 0; b < B; ++b) {
                    if (rows[b] == 0u) continue;
                    const uint32_t mine = rows[b] >> (4 * half); // this lane's rows: 8 (e / 4) + 4 half + e % 4
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        const u32x4_t finite = STRICT ? finite_bf16(w[b][j]) : w[b][j];
                        f32x16_t sum{};
                        if (exact) sum = mfma32<DT_BF16>(part[2], finite, sum);
                        sum = mfma32<DT_BF16>(part[1], finite, sum);
                        sum = mfma32<DT_BF16>(part[0], w[b][j], sum);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[I][j][e] += (mine >> (8 * (e >> 2) + (e & 3))) & 1u ? sum[e] : 0.0f;
                    }
                }
            }
        }
    });
}

template <bool QT, int HALF, int TM, int TN>
__device__ __forceinline__ void expand_adapters(const FusedArgs &a, f32x16_t (&acc)[TM][TN], int64_t r0, int64_t c0, int lane) {
    if (a.n <= 0 || a.r <= 0) return;
    expand_adapters_as<QT, HALF, false>(a, acc, r0, c0, lane);
    float all = 0.0f;                                            // a NaN where a sum is not finite
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) all = __builtin_fmaf(acc[i][j][e], 0.0f, all);
    if (__ballot(all != all) == 0u) return;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};
    expand_adapters_as<QT, HALF, true>(a, acc, r0, c0, lane);
}

}  // namespace gemm
