// mx_gemm.hip -- the products over block-scaled operands.
#include "mx_common.h"

namespace gemm {

__device__ __forceinline__ float mx_element(const MxArgs &a, MxOp op, int64_t row, int64_t col) {
    const uint32_t e = a.scales[row * a.ld_scales + col / kMxBlock];
    const uint8_t *const codes = static_cast<const uint8_t *>(a.g.B) + row * a.g.ldb;
    if (op == MX_DW) return float(int8_t(codes[col])) * mx_scale(e);
    const uint32_t pair = codes[col / 2];
    const uint32_t v = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(pair, mx4_scale(e), 0));
    return bf16_to_f32(col & 1 ? v >> 16 : v & 0xffffu);
}

// One thread per element of C.
template <int OP>
__global__ __launch_bounds__(256) void mx_element_kernel(MxArgs a) {
    const int64_t total = a.g.M * a.g.N, stride = int64_t(gridDim.x) * 256;
    const uint16_t *const A = static_cast<const uint16_t *>(a.g.A);
    for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < total; id += stride) {
        const int64_t i = id / a.g.N, j = id - i * a.g.N;
        float sum = 0.0f;
        for (int64_t k = 0; k < a.g.K; ++k) {
            const float x = bf16_to_f32(OP == MX_DW ? A[k * a.g.lda + i] : A[i * a.g.lda + k]);
            sum = fmaf(x, OP == MX_FWD ? mx_element(a, MX_FWD, j, k) : mx_element(a, MxOp(OP), k, j), sum);
        }
        write_c<DT_BF16>(a.g, i * a.g.ldc + j, sum);
    }
}

int launch_mx_gemm(const MxArgs &a, MxOp op, void *stream_ptr) {
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    const int64_t n = (a.g.M * a.g.N + 255) / 256;
    const dim3 grid(unsigned(n < (int64_t(1) << 20) ? n : (int64_t(1) << 20)));
    if (op == MX_FWD) hipLaunchKernelGGL(mx_element_kernel<MX_FWD>, grid, dim3(256), 0, stream, a);
    else if (op == MX_DX) hipLaunchKernelGGL(mx_element_kernel<MX_DX>, grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(mx_element_kernel<MX_DW>, grid, dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? LAUNCH_OK : LAUNCH_HIP_ERROR;
}

}  // namespace gemm
