"""A projection that many requests share, each with a low-rank adapter of its own, and its gradients.

    y_t = x_t W^T + s_i (x_t A_i^T) B_i^T       token t of a request with adapter i = index[t]; none where
                                                index[t] does not name one (-1)

The functions named like the C entry points of include/adapters_mi355x.h take plain integers and device
addresses.  The torch helpers read addresses, strides and the current stream and call them:

* ``linear_adapters(x, W, adapters, index)``: y, from one token up, tokens of the requests in any order;
* ``linear_adapters_dx(dy, W, adapters, index)``: the input gradient;
* ``linear_adapters_dw(x, dy, h, dh, index, n)``: every adapter's gradients, from what the two above leave with
  ``keep=True``.

``Adapters`` holds n adapters of one rank; one of a lower rank has zeros behind its own.  Ranks go up to 1024, a call's tokens to 2^26;
gradients are had of at most 65535 adapters at a time.  ``AdaptersLinear`` (feedforward.py) is the projection as a module.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

from . import binding as _b
from .mx import _ld

EXPORTED = ("adapters_linear_f32_bt", "adapters_linear_bf16_bt", "adapters_linear_f32", "adapters_linear_bf16", "adapters_dw_f32",
            "adapters_dw_bf16", "adapters_force_plan")
ADAPTERS_OP_FORWARD, ADAPTERS_OP_INPUT_GRADIENT = range(2)

_i64, _p, _int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int


class AdaptersSet(ctypes.Structure):
    _fields_ = [("n", _i64), ("r", _i64), ("A", _p), ("lda", _i64), ("sa", _i64), ("B", _p), ("ldb", _i64), ("sb", _i64), ("scale", _p)]


class Adapters(NamedTuple):
    """n adapters of rank r beside a weight of n_out x n_in: A (n x r x n_in) and B (n x n_out x r) in bf16, and n fp32
    scales (None: 1).  An adapter's rows may be strided, their elements may not."""
    A: "torch.Tensor"       # noqa: F821
    B: "torch.Tensor"       # noqa: F821
    scale: "torch.Tensor | None" = None     # noqa: F821


_LINEAR = [_i64] * 3 + [_p, _i64] * 2 + [ctypes.POINTER(AdaptersSet), _p] + [_p, _i64] + [_p, _p]
_DW = [_i64] * 5 + [_p, _i64] * 2 + [_p] * 3 + [_p, _i64, _i64] * 2 + [_p]
_fns = None


def lib():
    """The library's adapter entry points by name (raises if it has not been built)."""
    global _fns
    if _fns is None:
        l, fns = _b.lib(), {}
        for name in EXPORTED:
            fn = getattr(l, name)
            fn.restype = _int
            fn.argtypes = _LINEAR if "linear" in name else _DW if "dw" in name else [_int] * 3
            fns[name] = fn
        _fns = fns
    return _fns


def _linear(name):
    def call(M, N, K, X, ldx, W, ldw, adapters_set, index, Y, ldy, H=0, stream=0) -> int:
        return lib()[name](M, N, K, X or None, ldx, W or None, ldw, None if adapters_set is None else ctypes.byref(adapters_set),
                           index or None, Y or None, ldy, H or None, stream or None)
    call.__name__ = name
    return call


def _dw(name):
    def call(M, N, K, n, r, X, ldx, dY, lddy, H, dH, index, dA, ldda, sda, dB, lddb, sdb, stream=0) -> int:
        return lib()[name](M, N, K, n, r, X or None, ldx, dY or None, lddy, H or None, dH or None, index or None, dA or None, ldda, sda,
                           dB or None, lddb, sdb, stream or None)
    call.__name__ = name
    return call


adapters_linear_f32_bt, adapters_linear_bf16_bt, adapters_linear_f32, adapters_linear_bf16 = map(_linear, EXPORTED[:4])
adapters_dw_f32, adapters_dw_bf16 = map(_dw, EXPORTED[4:6])


def adapters_force_plan(op, config=-1, split_k=0) -> int:
    return lib()["adapters_force_plan"](op, config, split_k)


def _stack(x, n, rows, cols):
    """Row stride and stride from matrix to matrix of n matrices of rows x cols."""
    per, ld, step = x.stride()
    return _ld((ld, step), rows if n else 0, cols), per if n > 1 and rows and cols else rows * cols or 1


class _Helpers:
    def __init__(self):
        import torch
        fns = lib()
        bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
        raw_stream, empty, ok = torch._C._cuda_getCurrentRawStream, torch.empty, _b.GEMM_OK
        forward = {f32: fns["adapters_linear_f32_bt"], bf16: fns["adapters_linear_bf16_bt"]}
        backward = {f32: fns["adapters_linear_f32"], bf16: fns["adapters_linear_bf16"]}
        dws = {f32: fns["adapters_dw_f32"], bf16: fns["adapters_dw_bf16"]}

        current, device_of = torch._C._cuda_getDevice, torch.cuda.device

        def call(device, fn, *args):
            if current() == device:
                rc = fn(*args, raw_stream(device))
            else:                                           # the entry points work on the current device
                with device_of(device):
                    rc = fn(*args, raw_stream(device))
            if rc != ok:
                raise _b.GemmError(rc)

        def matrix(x, device=None):
            if x.dtype != bf16:
                raise TypeError("expected bfloat16 operands")
            if x.dim() != 2 or not x.is_cuda or (device is not None and x.get_device() != device):
                raise ValueError("expected matrices on one GPU")
            return x.shape

        def tokens_index(index, M, device):
            if index.dtype != i32:
                raise TypeError("the index is int32")
            if index.shape != (M,) or index.get_device() != device:
                raise ValueError("the index names one adapter a token, on the operands' GPU")
            if M > 1 and index.stride(0) != 1:
                raise ValueError("the index must be contiguous")
            return index.data_ptr()

        def linear(table, bt, X, W, adapters, index, out, out_dtype, keep):
            A, B, scale = adapters
            M, K = matrix(X)
            device = X.get_device()
            n_out, n_in = matrix(W, device)
            N, inner = (n_out, n_in) if bt else (n_in, n_out)
            if K != inner:
                raise ValueError("operand sizes do not fit")
            if A.dtype != bf16 or B.dtype != bf16 or (scale is not None and scale.dtype != f32):
                raise TypeError("adapters are bfloat16, their scales float32")
            if A.dim() != 3 or B.dim() != 3:
                raise ValueError("the adapters do not fit the weight")
            n, r = A.shape[:2]
            if A.shape[2] != n_in or B.shape != (n, n_out, r) or (scale is not None and scale.shape != (n,)):
                raise ValueError("the adapters do not fit the weight")
            if A.get_device() != device or B.get_device() != device or (scale is not None and scale.get_device() != device):
                raise ValueError("operands must be on the same GPU")
            if scale is not None and n > 1 and scale.stride(0) != 1:
                raise ValueError("the scales must be contiguous")
            where = tokens_index(index, M, device)
            dtype = out.dtype if out is not None else out_dtype or bf16
            if dtype not in table:
                raise TypeError("results are bfloat16 or float32")
            if out is None:
                out, ldy = empty(M, N, dtype=dtype, device=X.device), N or 1
            else:
                if out.shape != (M, N) or out.get_device() != device:
                    raise ValueError("bad output tensor")
                ldy = _ld(out.stride(), M, N)
            H = empty(M, r, dtype=f32, device=X.device) if keep else None
            held = AdaptersSet(n, r, A.data_ptr() or None, *_stack(A, n, r, n_in), B.data_ptr() or None, *_stack(B, n, n_out, r),
                               None if scale is None else scale.data_ptr() or None)
            call(device, table[dtype], M, N, K, X.data_ptr(), _ld(X.stride(), M, K), W.data_ptr(), _ld(W.stride(), n_out, n_in), held, where,
                 out.data_ptr(), ldy, H.data_ptr() if keep else None)
            return (out, H) if keep else out

        def weight_gradients(x, dy, h, dh, index, n, out_dtype):
            M, K = matrix(x)
            device = x.get_device()
            rows, N = matrix(dy, device)
            if h.dtype != f32 or dh.dtype != f32:
                raise TypeError("h and dh are float32")
            if rows != M or h.dim() != 2 or h.shape[0] != M or dh.shape != h.shape:
                raise ValueError("operand sizes do not fit")
            if h.get_device() != device or dh.get_device() != device:
                raise ValueError("operands must be on the same GPU")
            if not h.is_contiguous() or not dh.is_contiguous():
                raise ValueError("h and dh must be contiguous")
            r = h.shape[1]
            where = tokens_index(index, M, device)
            dtype = out_dtype or f32
            if dtype not in dws:
                raise TypeError("results are bfloat16 or float32")
            dA, dB = empty(n, r, K, dtype=dtype, device=x.device), empty(n, N, r, dtype=dtype, device=x.device)
            call(device, dws[dtype], M, N, K, n, r, x.data_ptr(), _ld(x.stride(), M, K), dy.data_ptr(), _ld(dy.stride(), M, N), h.data_ptr(),
                 dh.data_ptr(), where, dA.data_ptr(), K or 1, r * K or 1, dB.data_ptr(), r or 1, N * r or 1)
            return dA, dB

        self.forward = lambda *args: linear(forward, True, *args)
        self.backward = lambda *args: linear(backward, False, *args)
        self.weight_gradients = weight_gradients


_helpers = None


def _h():
    global _helpers
    if _helpers is None:
        _helpers = _Helpers()
    return _helpers


def linear_adapters(x, W, adapters: Adapters, index, out=None, out_dtype=None, keep=False):
    """y = x . W^T and each token's adapter's part (M x N, bf16 unless out_dtype or out says float32): x M x K, W N x K,
    index M int32.  With ``keep`` (y, h): h = s_i x . A_i^T (M x r, fp32), for ``linear_adapters_dw``."""
    return (_helpers or _h()).forward(x, W, adapters, index, out, out_dtype, keep)


def linear_adapters_dx(dy, W, adapters: Adapters, index, out=None, out_dtype=None, keep=False):
    """dx = dy . W and each token's adapter's part (M x N, bf16 unless out_dtype or out says float32): dy M x K, W K x N.
    With ``keep`` (dx, dh): dh = s_i dy . B_i (M x r, fp32), for ``linear_adapters_dw``."""
    return (_helpers or _h()).backward(dy, W, adapters, index, out, out_dtype, keep)


def linear_adapters_dw(x, dy, h, dh, index, n, out_dtype=None):
    """(dA, dB) of n adapters (n x r x n_in and n x n_out x r), fp32 unless out_dtype says bfloat16, from tokens' x and dy
    and the h and dh that ``linear_adapters`` and ``linear_adapters_dx`` kept.  An adapter without tokens gets zeros."""
    return (_helpers or _h()).weight_gradients(x, dy, h, dh, index, n, out_dtype)


def __getattr__(name):
    # The module, which needs torch at its definition.
    if name == "AdaptersLinear":
        from .feedforward import AdaptersLinear
        return AdaptersLinear
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
