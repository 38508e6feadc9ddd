// mx_common.h -- device helpers of the block-scaled kernels.
//
// E2M1 codes become bf16 values (and back) in the gfx950 conversion instructions, two
// elements at a time, the block's scale included.  Over all 256 code pairs and 256 scale
// bytes they give the exact value, subnormal results and the NaN of byte 255 among them,
// and over all finite bf16 inputs the nearest code, ties to even, saturated.
#pragma once

#include "gemm_common.h"
#include "mx.h"

namespace gemm {

typedef unsigned u32x4_any_mx __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned u32x2_any_mx __attribute__((ext_vector_type(2), aligned(1)));
typedef unsigned u32_any_mx __attribute__((aligned(1)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// A value that is the same in every lane, as a scalar: the compiler may form the uniform operands of
// a buffer resource on the vector unit, which the inline-assembly loads cannot take.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return uint32_t(__builtin_amdgcn_readfirstlane(int(v))); }
__device__ __forceinline__ const uint8_t *uniform(const uint8_t *p) {
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const uint8_t *>(uint64_t(uniform(uint32_t(at))) | (uint64_t(uniform(uint32_t(at >> 32))) << 32));
}

// The scale operand of the conversions for scale byte e: they use its exponent field.
__device__ __forceinline__ float mx4_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// Eight 4-bit codes (element i in bits 4 i) to eight bf16 values, two to a dword.
__device__ __forceinline__ u32x4_t mx4_to_bf16(uint32_t codes, float scale) {
    return u32x4_t{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// The first n of a block's 32 codes, zeros after them.
__device__ __forceinline__ u32x4_t mx4_first(u32x4_t codes, int n) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int left = n - 8 * t;
        codes[t] &= left >= 8 ? ~0u : left > 0 ? (1u << (4 * left)) - 1u : 0u;
    }
    return codes;
}

// 2^(e - 127) as fp32; NaN for e = 255.
__device__ __forceinline__ float mx_scale(uint32_t e) {
    return __builtin_bit_cast(float, e == 0u ? 0x00400000u : e == 255u ? 0x7fc00000u : e << 23);
}

// Four int8 codes (element i in byte i) times a scale to four bf16 values.  A code has seven
// significant bits and the scale one, so the product is a bf16 number and its upper half
// all of it.
__device__ __forceinline__ u32x2_t mx8_to_bf16(uint32_t codes, float scale) {
    const float f0 = float(int8_t(codes)) * scale, f1 = float(int8_t(codes >> 8)) * scale;
    const float f2 = float(int8_t(codes >> 16)) * scale, f3 = float(int8_t(codes >> 24)) * scale;
    return u32x2_t{perm(__builtin_bit_cast(uint32_t, f1), __builtin_bit_cast(uint32_t, f0), 0x07060302u),
                   perm(__builtin_bit_cast(uint32_t, f3), __builtin_bit_cast(uint32_t, f2), 0x07060302u)};
}

// ---------------------------------------------------------------------------
// K slices.  Each slice of an output tile leaves its partial sums in the workspace as its
// registers hold them, four floats of a thread at a time: slot v of thread t of slice s of
// the tile at 16 ((s SLOTS + v) THREADS + t), so that every access is a run of 1 KiB per wave
// (element by element, into rows of C's shape, the sums of 64 x 4096 in two slices took 6 us
// more).  The slice that arrives last adds the tile's slices up in their order, whichever
// it is, so the result does not depend on it.
//
// The ordering is store_tile's (gemm_common.h): stores and loads at the device's coherence
// point (sc1), each thread's stores complete before the barrier ahead of the ticket, the
// loads issued after the ticket's answer.
// ---------------------------------------------------------------------------
constexpr int kCoherent = 16;        // the sc1 bit of a buffer access: device scope

__device__ __forceinline__ void mx_store_part(__amdgpu_buffer_rsrc_t r, uint32_t off, f32x4_t v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, int(off), 0, kCoherent);
}
__device__ __forceinline__ f32x4_t mx_load_part(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, int(off), 0, kCoherent));
}

// The workspace of output tile `tile`: split_k slices of `slice_bytes`.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_parts(const KernelArgs &g, int tile, uint32_t slice_bytes) {
    uint8_t *const base = static_cast<uint8_t *>(g.workspace) + int64_t(tile) * g.split_k * slice_bytes;
    return make_rsrc(base, uint32_t(g.split_k) * slice_bytes);
}

// After a thread's partial stores: true in every thread of the slice that arrives last.
// `flag`: a word of LDS that nothing else uses.
__device__ __forceinline__ bool mx_last_slice(const KernelArgs &g, int tile, int &flag) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
        flag = __hip_atomic_fetch_add(&g.counters[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) ==
               unsigned(g.split_k - 1);
    __syncthreads();
    return flag != 0;
}
__device__ __forceinline__ void mx_reset_counter(const KernelArgs &g, int tile) {
    if (threadIdx.x == 0) __hip_atomic_store(&g.counters[tile], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// store_tile for the tile kernels: the last slice's sum as above; whole K, and slices that a
// kernel of its own adds up, as store_tile does.  Called by every thread of the workgroup;
// `holds` says whether this one's registers hold results (the workgroup's first BM x BN / (TM
// TN 16) threads do).  Rows past M are neither left in the workspace nor fetched.
template <int BM, int BN, int TM, int TN>
__device__ __forceinline__ void mx_store_tile(const KernelArgs &g, f32x16_t (&acc)[TM][TN], int tm, int tn, int slice,
                                              int64_t r0, int64_t c0, int lane, bool holds, int &flag) {
    KernelArgs out = g;
    if (g.split_k > 1 && g.reduce_in_kernel == REDUCE_LAST_SLICE) {
        const int64_t rows = holds ? g.M - r0 : 0;        // slot q of fragment row i: rows 32 i + 8 q .. + 7
        constexpr int THREADS = 64 * (BM / (32 * TM)) * (BN / (32 * TN));
        constexpr uint32_t SLICE = uint32_t(BM) * BN * 4;
        const int tile = tm * g.tiles_n + tn;
        const __amdgpu_buffer_rsrc_t parts = mx_parts(g, tile, SLICE);
        const uint32_t off = threadIdx.x * 16;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (32 * i + 8 * q >= rows) continue;
                    const f32x4_t v{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                    mx_store_part(parts, slice * SLICE + off + uint32_t(((i * TN + j) * 4 + q) * THREADS) * 16, v);
                }
        if (!mx_last_slice(g, tile, flag)) return;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = f32x16_t{};
        // Small tiles fetch four slices at once, eight where no more than 16 rows hold results (slots
        // 0 and 1 of the only fragment row): one after the other, each waits out a trip to
        // the coherence point.
        auto add = [&](int s, auto n_c, auto q_c) __attribute__((always_inline)) {
            constexpr int COUNT = decltype(n_c)::value, Q = decltype(q_c)::value;
            f32x4_t v[COUNT][TM][TN][Q];
#pragma unroll
            for (int u = 0; u < COUNT; ++u)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < Q; ++q)
                            v[u][i][j][q] = mx_load_part(parts, 32 * i + 8 * q < rows ? (s + u) * SLICE + off + uint32_t(((i * TN + j) * 4 + q) * THREADS) * 16 : kOOB);
#pragma unroll
            for (int u = 0; u < COUNT; ++u)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < Q; ++q)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += v[u][i][j][q][e];
        };
        constexpr int G = TM * TN >= 4 ? 1 : 4 / (TM * TN);
        using I1 = std::integral_constant<int, 1>;
        using I2 = std::integral_constant<int, 2>;
        using I4 = std::integral_constant<int, 4>;
        int s = 0;
        if (TM * TN == 1 && rows <= 16)
            for (; s + 8 <= g.split_k; s += 8) add(s, std::integral_constant<int, 8>{}, I2{});
        for (; s + G <= g.split_k; s += G) add(s, std::integral_constant<int, G>{}, I4{});
        for (; s < g.split_k; ++s) add(s, I1{}, I4{});
        mx_reset_counter(g, tile);
        out.split_k = 1;
    }
    if (holds) store_tile<DT_BF16, BM, BN, TM, TN>(out, acc, tm, tn, slice, r0, c0, lane, flag);
}

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

}  // namespace gemm
