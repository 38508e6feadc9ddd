// mx_pack.hip -- packing bf16 matrices to block-scaled codes and back.
//
// A thread holds eight consecutive elements of a row, four neighbouring threads one block
// of 32: bf16 is read and written 16 bytes per thread, codes 4 or 8 bytes, all contiguous
// across the wave.  The largest magnitude of a block is the largest of its bit patterns
// without their signs (infinities and NaN above every finite one), so its power of two is
// that pattern's exponent field and no logarithm is taken.
//
// Bound by memory: 2.5 to 3 bytes move per element and both conversions are a handful of
// instructions for it.  14336 x 4096 to 4 bits and back: 30.9 and 23.5 us (4.8 and 6.3 TB/s; a
// large copy moves 4.8, and the second finds part of the codes in the cache); 2048 x 11008 to 8
// bits and back: 14.4 and 13.1 us.
#include "mx_common.h"

namespace gemm {

// Where thread `id` works: row and first column of its eight elements, false past the end.
// A row has four threads for each of its blocks, the last block's too.
struct MxPlace {
    int64_t row, col;
    int left;              // elements of the row from col on, at most 8 (may be <= 0 in the last block)
};
__device__ __forceinline__ MxPlace mx_place(const MxMatrixArgs &a, int64_t id, int64_t groups) {
    MxPlace p;
    if (id >> 32 == 0 && groups >> 32 == 0) {       // almost always: 32-bit division
        const uint32_t r = uint32_t(id) / uint32_t(groups);
        p.row = r;
        p.col = int64_t(uint32_t(id) - r * uint32_t(groups)) * 8;
    } else {
        p.row = id / groups;
        p.col = (id - p.row * groups) * 8;
    }
    const int64_t left = a.cols - p.col;
    p.left = left < 8 ? int(left) : 8;
    return p;
}

template <int BITS>
__global__ __launch_bounds__(256) void mx_pack_kernel(MxMatrixArgs a, int64_t groups, int64_t total) {
    const int64_t stride = int64_t(gridDim.x) * 256;
    // `total` is a multiple of four: the four threads of a block are in or out together.
    for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < total; id += stride) {
        const MxPlace p = mx_place(a, id, groups);
        const uint16_t *const src = static_cast<const uint16_t *>(a.x) + p.row * a.ldx + p.col;
        u32x4_t v{0u, 0u, 0u, 0u};
        if (p.left == 8) {
            v = *reinterpret_cast<const u32x4_any_mx *>(src);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < p.left) v[i / 2] |= uint32_t(src[i]) << (16 * (i & 1));
        }
        uint32_t big = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = v[i] & 0x7fffu, hi = (v[i] >> 16) & 0x7fffu;
            big = big > lo ? big : lo;
            big = big > hi ? big : hi;
        }
        // Over the block's four threads: quad permutations that exchange neighbours, then pairs.
        uint32_t other = dpp_quad<0xB1>(big);
        big = big > other ? big : other;
        other = dpp_quad<0x4E>(big);
        big = big > other ? big : other;
        const uint32_t ex = big >> 7, top = BITS == 4 ? 2u : 6u;
        const bool fine = ex != 255u;
        const uint32_t e = !fine ? 255u : ex > top ? ex - top : 0u;
        if (p.left > 0 && (threadIdx.x & 3) == 0) a.scales[p.row * a.ld_scales + p.col / kMxBlock] = uint8_t(e);
        if constexpr (BITS == 4) {
            uint32_t c = 0;
            const float s = mx4_scale(e);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, uint32_t(v[0])), s, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, uint32_t(v[1])), s, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, uint32_t(v[2])), s, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, uint32_t(v[3])), s, 3);
            if (!fine) c = 0;
            uint8_t *const dst = static_cast<uint8_t *>(a.codes) + p.row * a.ldq + p.col / 2;
            if (p.left == 8) {
                *reinterpret_cast<u32_any_mx *>(dst) = c;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (2 * i < p.left) dst[i] = uint8_t(c >> (8 * i));
            }
        } else {
            // x / 2^(e - 127), exact in fp32; the sum with 1.5 * 2^23 rounds it to the nearest
            // integer, ties to even, and leaves that integer in its low byte.
            const float inv = __builtin_bit_cast(float, (254u - (fine ? e : 127u)) << 23);
            uint32_t q[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = bf16_to_f32((v[i / 2] >> (16 * (i & 1))) & 0xffffu) * inv;
                q[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(x, -127.0f, 127.0f) + 12582912.0f) & 0xffu;
            }
            u32x2_t c{q[0] | (q[1] << 8) | (q[2] << 16) | (q[3] << 24), q[4] | (q[5] << 8) | (q[6] << 16) | (q[7] << 24)};
            if (!fine) c = u32x2_t{0u, 0u};
            uint8_t *const dst = static_cast<uint8_t *>(a.codes) + p.row * a.ldq + p.col;
            if (p.left == 8) {
                *reinterpret_cast<u32x2_any_mx *>(dst) = c;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < p.left) dst[i] = uint8_t(c[i / 4] >> (8 * (i & 3)));
            }
        }
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void mx_unpack_kernel(MxMatrixArgs a, int64_t groups, int64_t total) {
    const int64_t stride = int64_t(gridDim.x) * 256;
    for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < total; id += stride) {
        const MxPlace p = mx_place(a, id, groups);
        if (p.left <= 0) continue;
        const uint32_t e = a.scales[p.row * a.ld_scales + p.col / kMxBlock];
        const uint8_t *const src = static_cast<const uint8_t *>(a.codes) + p.row * a.ldq + (BITS == 4 ? p.col / 2 : p.col);
        u32x4_t v;
        if constexpr (BITS == 4) {
            uint32_t c = 0;
            if (p.left == 8) {
                c = *reinterpret_cast<const u32_any_mx *>(src);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (2 * i < p.left) c |= uint32_t(src[i]) << (8 * i);
            }
            v = mx4_to_bf16(c, mx4_scale(e));
        } else {
            u32x2_t c{0u, 0u};
            if (p.left == 8) {
                c = *reinterpret_cast<const u32x2_any_mx *>(src);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < p.left) c[i / 4] |= uint32_t(src[i]) << (8 * (i & 3));
            }
            const float s = mx_scale(e);
            const u32x2_t lo = mx8_to_bf16(c[0], s), hi = mx8_to_bf16(c[1], s);
            v = u32x4_t{lo[0], lo[1], hi[0], hi[1]};
        }
        uint16_t *const dst = static_cast<uint16_t *>(a.x) + p.row * a.ldx + p.col;
        if (p.left == 8) {
            *reinterpret_cast<u32x4_any_mx *>(dst) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < p.left) dst[i] = uint16_t(v[i / 2] >> (16 * (i & 1)));
        }
    }
}

static int64_t mx_groups(const MxMatrixArgs &a) { return (a.cols + kMxBlock - 1) / kMxBlock * 4; }
static unsigned mx_grid(int64_t total) {
    const int64_t n = (total + 255) / 256;
    return unsigned(n < (int64_t(1) << 20) ? n : (int64_t(1) << 20));
}

int launch_mx_pack(const MxMatrixArgs &a, int bits, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    const int64_t groups = mx_groups(a), total = groups * a.rows;
    if (bits == 4) hipLaunchKernelGGL(mx_pack_kernel<4>, dim3(mx_grid(total)), dim3(256), 0, stream, a, groups, total);
    else hipLaunchKernelGGL(mx_pack_kernel<8>, dim3(mx_grid(total)), dim3(256), 0, stream, a, groups, total);
    return hipGetLastError() == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

int launch_mx_unpack(const MxMatrixArgs &a, int bits, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    const int64_t groups = mx_groups(a), total = groups * a.rows;
    if (bits == 4) hipLaunchKernelGGL(mx_unpack_kernel<4>, dim3(mx_grid(total)), dim3(256), 0, stream, a, groups, total);
    else hipLaunchKernelGGL(mx_unpack_kernel<8>, dim3(mx_grid(total)), dim3(256), 0, stream, a, groups, total);
    return hipGetLastError() == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

}  // namespace gemm
