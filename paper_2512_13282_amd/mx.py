"""Block-scaled operands: linear layers over 4-bit weights, activation checkpoints in 8 bits.

The functions named like the C entry points of include/mx_mi355x.h (``mx_pack4``, ...) take
plain integers and device addresses.  The torch helpers read addresses, strides and the
current stream and call them:

* ``pack_mx4(W)`` / ``pack_mx8(X)``: a bf16 matrix as an ``MxMatrix`` (codes, a scale byte for
  every 32 elements of a row); ``unpack_mx(Q)``: the bf16 matrix it stands for, exactly;
* ``linear_mx4(A, W)``: A . W^T over a packed weight W (N x K), from one row up;
* ``linear_mx4_dx(dY, W)``: its input gradient dY . W over the same packed weight (``dY`` has
  the weight's rows as its columns);
* ``linear_mx8_dw(dY, X)``: the weight gradient dY^T . X over a packed input X (tokens x in).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from . import binding as _b

EXPORTED = ("mx_pack4", "mx_pack8", "mx_unpack4", "mx_unpack8",
            "mx_gemm_bf16_mx4_f32_bt", "mx_gemm_bf16_mx4_bf16_bt", "mx_gemm_bf16_mx4_f32",
            "mx_gemm_bf16_mx4_bf16", "mx_gemm_bf16_mx8_f32_at", "mx_gemm_bf16_mx8_bf16_at",
            "mx_plan", "mx_force_plan")
BLOCK = 32
MX_OP_FORWARD, MX_OP_INPUT_GRADIENT, MX_OP_WEIGHT_GRADIENT = range(3)


class PlanInfo(ctypes.Structure):
    _fields_ = [("config", ctypes.c_int32), ("bm", ctypes.c_int32), ("bn", ctypes.c_int32),
                ("split_k", ctypes.c_int32), ("k_chunk", ctypes.c_int64), ("name", ctypes.c_char * 48)]


_fns = None


def lib():
    """The library's block-scaled entry points by name (raises if it has not been built)."""
    global _fns
    if _fns is None:
        l = _b.lib()
        i64, p = ctypes.c_int64, ctypes.c_void_p
        fns = {}
        for name in EXPORTED:
            fn = getattr(l, name)
            fn.restype = ctypes.c_int
            fn.argtypes = [i64, i64, i64, p, i64, p, i64, p, i64, p, i64, p] if "gemm" in name else \
                [i64, i64, p, i64, p, i64, p, i64, p]
            fns[name] = fn
        fns["mx_plan"].argtypes = [ctypes.c_int, i64, i64, i64, ctypes.POINTER(PlanInfo)]
        fns["mx_force_plan"].argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int]
        _fns = fns
    return _fns


def _convert(name):
    def call(rows, cols, src, ld_src, dst, ld_dst, third, ld_third, stream=0) -> int:
        return lib()[name](rows, cols, src or None, ld_src, dst or None, ld_dst, third or None, ld_third, stream or None)
    call.__name__ = name
    return call


def _product(name):
    def call(M, N, K, A, lda, codes, ldq, scales, lds, C, ldc, stream=0) -> int:
        return lib()[name](M, N, K, A or None, lda, codes or None, ldq, scales or None, lds, C or None, ldc,
                           stream or None)
    call.__name__ = name
    return call


mx_pack4, mx_pack8, mx_unpack4, mx_unpack8 = map(_convert, EXPORTED[:4])
(mx_gemm_bf16_mx4_f32_bt, mx_gemm_bf16_mx4_bf16_bt, mx_gemm_bf16_mx4_f32, mx_gemm_bf16_mx4_bf16,
 mx_gemm_bf16_mx8_f32_at, mx_gemm_bf16_mx8_bf16_at) = map(_product, EXPORTED[4:10])


def mx_plan(op, M, N, K) -> dict:
    """The plan of a product (MX_OP_*) as a dict; raises GemmError on a bad argument."""
    info = PlanInfo()
    rc = lib()["mx_plan"](op, M, N, K, ctypes.byref(info))
    if rc != _b.GEMM_OK:
        raise _b.GemmError(rc)
    return {f: getattr(info, f) for f, _ in PlanInfo._fields_} | {"name": info.name.decode()}


def mx_force_plan(op, config=-1, split_k=0) -> int:
    return lib()["mx_force_plan"](op, config, split_k)


class MxMatrix(NamedTuple):
    """A packed matrix of ``codes.shape[0]`` rows and ``cols`` columns: uint8 codes hold two 4-bit
    elements each (rows x ceil(cols / 2)), int8 codes one (rows x cols); uint8 scales are rows x
    ceil(cols / 32).  Rows may be strided, their elements may not."""
    codes: "torch.Tensor"   # noqa: F821
    scales: "torch.Tensor"  # noqa: F821
    cols: int


def _row_stride(t):
    """The row stride of a matrix whose rows are contiguous (a single row or column has no
    meaningful other stride)."""
    rows, cols = t.shape
    ld, step = t.stride()
    if step != 1 and cols > 1:
        raise ValueError("rows must be contiguous")
    return max(ld, cols, 1) if rows > 1 else max(cols, 1)


def _check_packed(Q, torch, bits, device):
    codes, scales, cols = Q
    if codes.dtype != (torch.uint8 if bits == 4 else torch.int8) or scales.dtype != torch.uint8:
        raise TypeError(f"expected {bits}-bit codes with uint8 scales")
    if codes.dim() != 2 or scales.dim() != 2 or codes.shape[1] != ((cols + 1) // 2 if bits == 4 else cols) \
            or scales.shape != (codes.shape[0], -(-cols // BLOCK)):
        raise ValueError("codes and scales do not fit the matrix")
    if not codes.is_cuda or codes.get_device() != device or scales.get_device() != device:
        raise ValueError("operands must be on the same GPU")


def _pack(X, bits):
    import torch
    if X.dtype != torch.bfloat16:
        raise TypeError("expected a bfloat16 matrix")
    if X.dim() != 2 or not X.is_cuda:
        raise ValueError("expected a matrix on the GPU")
    rows, cols = X.shape
    ldx = _row_stride(X)
    nbytes, blocks = ((cols + 1) // 2 if bits == 4 else cols), -(-cols // BLOCK)
    # Rows at a stride of whole 16 bytes: what the products read in aligned pieces.
    ldq = -(-nbytes // 16) * 16
    codes = torch.empty((rows, ldq), dtype=torch.uint8 if bits == 4 else torch.int8, device=X.device)[:, :nbytes]
    scales = torch.empty((rows, blocks), dtype=torch.uint8, device=X.device)
    rc = (mx_pack4 if bits == 4 else mx_pack8)(rows, cols, X.data_ptr(), ldx, codes.data_ptr(), max(ldq, 1),
                                               scales.data_ptr(), max(blocks, 1),
                                               torch._C._cuda_getCurrentRawStream(X.get_device()))
    if rc != _b.GEMM_OK:
        raise _b.GemmError(rc)
    return MxMatrix(codes, scales, cols)


def pack_mx4(X) -> MxMatrix:
    """A bf16 matrix packed to 4-bit elements, a scale for every 32 of a row."""
    return _pack(X, 4)


def pack_mx8(X) -> MxMatrix:
    """A bf16 matrix packed to 8-bit elements, a scale for every 32 of a row."""
    return _pack(X, 8)


def unpack_mx(Q, out=None):
    """The bf16 matrix that a packed one stands for, exactly."""
    import torch
    codes, scales, cols = Q
    bits = 8 if codes.dtype == torch.int8 else 4
    _check_packed(Q, torch, bits, codes.get_device())
    rows = codes.shape[0]
    if out is None:
        out = torch.empty((rows, cols), dtype=torch.bfloat16, device=codes.device)
    elif out.dtype != torch.bfloat16 or out.shape != (rows, cols) or out.get_device() != codes.get_device():
        raise ValueError("bad output tensor")
    rc = (mx_unpack4 if bits == 4 else mx_unpack8)(rows, cols, codes.data_ptr(), _row_stride(codes), scales.data_ptr(),
                                                   _row_stride(scales), out.data_ptr(), _row_stride(out),
                                                   torch._C._cuda_getCurrentRawStream(codes.get_device()))
    if rc != _b.GEMM_OK:
        raise _b.GemmError(rc)
    return out


def _multiply(stem, bits, A, Q, M, N, K, inner, out, out_dtype):
    import torch
    if A.dtype != torch.bfloat16:
        raise TypeError("expected a bfloat16 operand")
    if not A.is_cuda:
        raise ValueError("operands must be on the same GPU")
    device = A.get_device()
    _check_packed(Q, torch, bits, device)
    if K != inner:
        raise ValueError("operand sizes do not fit")
    if out is None:
        if out_dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("results are bfloat16 or float32")
        out = torch.empty((M, N), dtype=out_dtype, device=A.device)
    elif out.dtype not in (torch.bfloat16, torch.float32) or out.shape != (M, N) or out.get_device() != device:
        raise ValueError("bad output tensor")
    fn = lib()[stem.format("f32" if out.dtype == torch.float32 else "bf16")]
    rc = fn(M, N, K, A.data_ptr(), _row_stride(A), Q.codes.data_ptr(), _row_stride(Q.codes), Q.scales.data_ptr(),
            _row_stride(Q.scales), out.data_ptr(), _row_stride(out), torch._C._cuda_getCurrentRawStream(device))
    if rc != _b.GEMM_OK:
        raise _b.GemmError(rc)
    return out


def _matrix(A):
    if A.dim() != 2:
        raise ValueError("expected a matrix")
    return A.shape


def linear_mx4(A, W, out=None, out_dtype=None):
    """A (M x K bf16) . W^T over a 4-bit weight W (N x K): M x N, bf16 unless out_dtype or out
    says float32."""
    import torch
    M, K = _matrix(A)
    return _multiply("mx_gemm_bf16_mx4_{}_bt", 4, A, W, M, W.codes.shape[0], K, W.cols, out, out_dtype or torch.bfloat16)


def linear_mx4_dx(dY, W, out=None, out_dtype=None):
    """dY (M x N bf16) . W over a 4-bit weight W (N x K): the input gradient, M x K, bf16 unless
    out_dtype or out says float32."""
    import torch
    M, N = _matrix(dY)
    return _multiply("mx_gemm_bf16_mx4_{}", 4, dY, W, M, W.cols, N, W.codes.shape[0], out, out_dtype or torch.bfloat16)


def linear_mx8_dw(dY, X, out=None, out_dtype=None):
    """dY^T . X over an 8-bit input X (tokens x K) and dY (tokens x N bf16): the weight gradient,
    N x K, fp32 unless out_dtype or out says bfloat16."""
    import torch
    T, N = _matrix(dY)
    return _multiply("mx_gemm_bf16_mx8_{}_at", 8, dY, X, N, X.cols, T, X.codes.shape[0], out, out_dtype or torch.float32)
