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

Operands may be strided along their rows.  An expanded one (the gradient of a sum over tokens, say)
is refused, as by the dense helpers: ``.contiguous()`` makes it one that is taken.
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


# The helpers' per-call work is what bounds the smallest calls (7 us of host beside 3 us of kernel), so
# each is bound once to torch and its entry points, asks each tensor for every property once and takes
# the stream's handle without a Stream object.

def _ld(stride, rows, cols):
    """The row stride of a matrix whose rows are contiguous (a column's elements are single, and a
    single row or an empty matrix has no meaningful stride).  The entry points refuse one that is
    shorter than a row: an expanded tensor's, say, which holds fewer elements than the matrix."""
    ld, step = stride
    if step != 1 and cols > 1 and rows:
        raise ValueError("rows must be contiguous")
    return ld if rows > 1 and cols else cols or 1


def _packed(Q, bits, code_dtype, byte_dtype, device):
    """(rows, cols, codes' address, row stride, scales' address, row stride) of a packed matrix."""
    codes, scales, cols = Q
    if codes.dtype != code_dtype or scales.dtype != byte_dtype:
        raise TypeError(f"expected {bits}-bit codes with uint8 scales")
    if codes.dim() != 2 or scales.dim() != 2:
        raise ValueError("codes and scales do not fit the matrix")
    rows, width = codes.shape
    blocks = (cols + 31) // 32
    if width != ((cols + 1) // 2 if bits == 4 else cols) or scales.shape != (rows, blocks):
        raise ValueError("codes and scales do not fit the matrix")
    if not codes.is_cuda or codes.get_device() != device or scales.get_device() != device:
        raise ValueError("operands must be on the same GPU")
    return (rows, cols, codes.data_ptr(), _ld(codes.stride(), rows, width), scales.data_ptr(),
            _ld(scales.stride(), rows, blocks))


def _pack_helper(bits):
    import torch
    fn = lib()[f"mx_pack{bits}"]
    bf16, byte, code_dtype = torch.bfloat16, torch.uint8, torch.uint8 if bits == 4 else torch.int8
    raw_stream, empty, ok = torch._C._cuda_getCurrentRawStream, torch.empty, _b.GEMM_OK
    empty_strided = torch.empty_strided

    def pack(X):
        if X.dtype != bf16:
            raise TypeError("expected a bfloat16 matrix")
        if X.dim() != 2 or not X.is_cuda:
            raise ValueError("expected a matrix on the GPU")
        rows, cols = X.shape
        width, blocks = ((cols + 1) // 2 if bits == 4 else cols), (cols + 31) // 32
        # Rows at a stride of whole 16 bytes: what the products read in aligned pieces.
        ldq = (width + 15) // 16 * 16
        device = X.device
        codes = empty_strided((rows, width), (ldq, 1), dtype=code_dtype, device=device)
        scales = empty(rows, blocks, dtype=byte, device=device)
        rc = fn(rows, cols, X.data_ptr(), _ld(X.stride(), rows, cols), codes.data_ptr(), ldq or 1, scales.data_ptr(),
                blocks or 1, raw_stream(X.get_device()))
        if rc != ok:
            raise _b.GemmError(rc)
        return MxMatrix(codes, scales, cols)

    return pack


def _unpack_helper():
    import torch
    fns = {torch.uint8: (lib()["mx_unpack4"], 4), torch.int8: (lib()["mx_unpack8"], 8)}
    bf16, byte = torch.bfloat16, torch.uint8
    raw_stream, empty, ok = torch._C._cuda_getCurrentRawStream, torch.empty, _b.GEMM_OK

    def unpack(Q, out):
        code_dtype = Q.codes.dtype
        if code_dtype not in fns:
            raise TypeError("expected uint8 (4-bit) or int8 (8-bit) codes")
        fn, bits = fns[code_dtype]
        device = Q.codes.get_device()
        rows, cols, codes, ldq, scales, lds = _packed(Q, bits, code_dtype, byte, device)
        if out is None:
            out = empty(rows, cols, dtype=bf16, device=Q.codes.device)
        elif out.dtype != bf16 or out.shape != (rows, cols) or out.get_device() != device:
            raise ValueError("bad output tensor")
        rc = fn(rows, cols, codes, ldq, scales, lds, out.data_ptr(), _ld(out.stride(), rows, cols), raw_stream(device))
        if rc != ok:
            raise _b.GemmError(rc)
        return out

    return unpack


def _product_helper(op):
    import torch
    stem, bits = {MX_OP_FORWARD: ("mx_gemm_bf16_mx4_{}_bt", 4), MX_OP_INPUT_GRADIENT: ("mx_gemm_bf16_mx4_{}", 4),
                  MX_OP_WEIGHT_GRADIENT: ("mx_gemm_bf16_mx8_{}_at", 8)}[op]
    bf16, byte, code_dtype = torch.bfloat16, torch.uint8, torch.uint8 if bits == 4 else torch.int8
    fns = {torch.float32: lib()[stem.format("f32")], bf16: lib()[stem.format("bf16")]}
    raw_stream, empty, ok = torch._C._cuda_getCurrentRawStream, torch.empty, _b.GEMM_OK
    default = torch.float32 if op == MX_OP_WEIGHT_GRADIENT else bf16

    def multiply(A, Q, out, out_dtype):
        if A.dtype != bf16:
            raise TypeError("expected a bfloat16 operand")
        if A.dim() != 2 or not A.is_cuda:
            raise ValueError("expected a matrix on the GPU")
        device = A.get_device()
        b_rows, b_cols, codes, ldq, scales, lds = _packed(Q, bits, code_dtype, byte, device)
        rows, cols = A.shape
        if op == MX_OP_FORWARD:
            M, K, N, inner = rows, cols, b_rows, b_cols
        else:
            inner, N = b_rows, b_cols
            M, K = (rows, cols) if op == MX_OP_INPUT_GRADIENT else (cols, rows)
        if K != inner:
            raise ValueError("operand sizes do not fit")
        if out is None:
            out_dtype = out_dtype or default
            if out_dtype not in fns:
                raise TypeError("results are bfloat16 or float32")
            out = empty(M, N, dtype=out_dtype, device=A.device)
            ldc = N or 1
        else:
            out_dtype = out.dtype
            if out_dtype not in fns or out.shape != (M, N) or out.get_device() != device:
                raise ValueError("bad output tensor")
            ldc = _ld(out.stride(), M, N)
        rc = fns[out_dtype](M, N, K, A.data_ptr(), _ld(A.stride(), rows, cols), codes, ldq, scales, lds, out.data_ptr(),
                            ldc, raw_stream(device))
        if rc != ok:
            raise _b.GemmError(rc)
        return out

    return multiply


_bound = {}


def _helper(key, make, *args):
    fn = _bound.get(key)
    if fn is None:
        fn = _bound[key] = make(*args)
    return fn


def pack_mx4(X) -> MxMatrix:
    """A bf16 matrix packed to 4-bit elements, a scale for every 32 of a row."""
    return (_bound.get("pack4") or _helper("pack4", _pack_helper, 4))(X)


def pack_mx8(X) -> MxMatrix:
    """A bf16 matrix packed to 8-bit elements, a scale for every 32 of a row."""
    return (_bound.get("pack8") or _helper("pack8", _pack_helper, 8))(X)


def unpack_mx(Q, out=None):
    """The bf16 matrix that a packed one stands for, exactly."""
    return (_bound.get("unpack") or _helper("unpack", _unpack_helper))(Q, out)


def linear_mx4(A, W, out=None, out_dtype=None):
    """A (M x K bf16) . W^T over a 4-bit weight W (N x K): M x N, bf16 unless out_dtype or out
    says float32."""
    return (_bound.get(0) or _helper(0, _product_helper, MX_OP_FORWARD))(A, W, out, out_dtype)


def linear_mx4_dx(dY, W, out=None, out_dtype=None):
    """dY (M x N bf16) . W over a 4-bit weight W (N x K): the input gradient, M x K, bf16 unless
    out_dtype or out says float32."""
    return (_bound.get(1) or _helper(1, _product_helper, MX_OP_INPUT_GRADIENT))(dY, W, out, out_dtype)


def linear_mx8_dw(dY, X, out=None, out_dtype=None):
    """dY^T . X over an 8-bit input X (tokens x K) and dY (tokens x N bf16): the weight gradient,
    N x K, fp32 unless out_dtype or out says bfloat16."""
    return (_bound.get(2) or _helper(2, _product_helper, MX_OP_WEIGHT_GRADIENT))(dY, X, out, out_dtype)
