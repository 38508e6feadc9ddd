"""The gated feed-forward block: H = act(X Wg^T) * (X Wu^T), Y = H Wd^T, and its gradients.

The functions named like the C entry points of include/ffn_mi355x.h (``ffn_gated_bf16_bt``, ...) take
plain integers and device addresses.  The torch helpers read addresses, strides and the
current stream and call them:

* ``gated_linear(X, Wg, Wu)``: H, and with ``keep=True`` the bf16 G and U that the backward pass takes;
* ``gated_linear_grad(dY, Wd, G, U)``: the gradients of G and U, and H again, from the block's output gradient;
* ``gated_linear_bwd(dH, G, U)``: the gradients of G and U from that of H, where something else follows;
* ``gated_linear_dx(dG, Wg, dU, Wu)``: the input gradient;
* ``gated_linear_dw(dG, dU, X)``: both weight gradients, and ``linear_dw(dY, X)`` one projection's;
* ``GatedLinear`` and ``GatedFeedForward`` (feedforward.py): H and the whole block as modules, with all of them behind
  autograd.

Weights are laid out as torch's linear layers have them (outputs x inputs).  Operands are bf16
matrices, which may be strided along their rows; an expanded one is refused, as by the dense helpers.
"""
from __future__ import annotations

import ctypes

from . import binding as _b
from .mx import _ld

EXPORTED = ("ffn_gated_bf16_bt", "ffn_gated_grad_bf16", "ffn_gated_bwd_bf16", "ffn_gated_dx_f32", "ffn_gated_dx_bf16", "ffn_gated_dw_f32",
            "ffn_gated_dw_bf16", "ffn_dw_f32", "ffn_dw_bf16", "ffn_plan", "ffn_force_plan")
ACTIVATIONS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}
FFN_OP_GATED, FFN_OP_GRAD, FFN_OP_DX, FFN_OP_GATED_DW, FFN_OP_DW = range(5)

_i64, _p, _int = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
_matrix = [_p, _i64]


class PlanInfo(ctypes.Structure):
    _fields_ = [("config", ctypes.c_int32), ("bm", ctypes.c_int32), ("bn", ctypes.c_int32),
                ("split_k", ctypes.c_int32), ("k_chunk", ctypes.c_int64), ("name", ctypes.c_char * 48)]


_ARGS = {
    "ffn_gated_bf16_bt": [_i64] * 3 + _matrix * 3 + [_int] + _matrix * 3 + [_p],
    "ffn_gated_grad_bf16": [_i64] * 3 + _matrix * 4 + [_int] + _matrix * 3 + [_p],
    "ffn_gated_bwd_bf16": [_i64] * 2 + _matrix * 3 + [_int] + _matrix * 2 + [_p],
    **{f"ffn_gated_dx_{t}": [_i64] * 3 + _matrix * 5 + [_p] for t in ("f32", "bf16")},
    **{f"ffn_gated_dw_{t}": [_i64] * 3 + _matrix * 5 + [_p] for t in ("f32", "bf16")},
    **{f"ffn_dw_{t}": [_i64] * 3 + _matrix * 3 + [_p] for t in ("f32", "bf16")},
    "ffn_plan": [_int, _i64, _i64, _i64, ctypes.POINTER(PlanInfo)],
    "ffn_force_plan": [_int, _int, _int],
}
_fns = None


def lib():
    """The library's feed-forward entry points by name (raises if it has not been built)."""
    global _fns
    if _fns is None:
        l, fns = _b.lib(), {}
        for name in EXPORTED:
            fn = getattr(l, name)
            fn.restype, fn.argtypes = _int, _ARGS[name]
            fns[name] = fn
        _fns = fns
    return _fns


def _entry(name):
    def call(*args) -> int:
        # The stream may be left out; addresses of 0 are NULL.
        types = _ARGS[name]
        args = args + (0,) * (len(types) - len(args) if len(args) == len(types) - 1 else 0)
        return lib()[name](*((a or None) if t is _p else a for a, t in zip(args, types, strict=True)))
    call.__name__ = name
    return call


(ffn_gated_bf16_bt, ffn_gated_grad_bf16, ffn_gated_bwd_bf16, ffn_gated_dx_f32, ffn_gated_dx_bf16, ffn_gated_dw_f32, ffn_gated_dw_bf16,
 ffn_dw_f32, ffn_dw_bf16) = map(_entry, EXPORTED[:9])


def ffn_plan(op, M, N, K) -> dict:
    """The plan of a call (FFN_OP_*) as a dict; raises GemmError on a bad argument."""
    info = PlanInfo()
    rc = lib()["ffn_plan"](op, M, N, K, ctypes.byref(info))
    if rc != _b.GEMM_OK:
        raise _b.GemmError(rc)
    return {f: getattr(info, f) for f, _ in PlanInfo._fields_} | {"name": info.name.decode()}


def ffn_force_plan(op, config=-1, split_k=0) -> int:
    return lib()["ffn_force_plan"](op, config, split_k)


# Bound once to torch and the entry points, for the helpers' per-call work is what bounds the smallest calls.
class _Helpers:
    def __init__(self):
        import torch
        fns = lib()
        bf16, f32 = torch.bfloat16, torch.float32
        raw_stream, empty, ok = torch._C._cuda_getCurrentRawStream, torch.empty, _b.GEMM_OK
        dx = {f32: fns["ffn_gated_dx_f32"], bf16: fns["ffn_gated_dx_bf16"]}
        dw2 = {f32: fns["ffn_gated_dw_f32"], bf16: fns["ffn_gated_dw_bf16"]}
        dw1 = {f32: fns["ffn_dw_f32"], bf16: fns["ffn_dw_bf16"]}
        f_gated, f_grad = fns["ffn_gated_bf16_bt"], fns["ffn_gated_grad_bf16"]

        def operand(x, rows, cols, device):
            """Address and row stride of a bf16 matrix of rows x cols on `device`."""
            if x.dtype != bf16:
                raise TypeError("expected bfloat16 operands")
            if x.dim() != 2 or x.shape != (rows, cols):
                raise ValueError("operand sizes do not fit")
            if not x.is_cuda or x.get_device() != device:
                raise ValueError("operands must be on the same GPU")
            return x.data_ptr(), _ld(x.stride(), rows, cols)

        def matrix(x):
            if x.dtype != bf16:
                raise TypeError("expected bfloat16 operands")
            if x.dim() != 2 or not x.is_cuda:
                raise ValueError("expected a matrix on the GPU")
            return x.shape

        def result(out, rows, cols, dtype, like):
            """An output tensor, the caller's or a new one, with its address and row stride."""
            if out is None:
                out = empty(rows, cols, dtype=dtype, device=like.device)
                return out, out.data_ptr(), cols or 1
            if out.dtype != dtype or out.shape != (rows, cols) or not out.is_cuda or out.get_device() != like.get_device():
                raise ValueError("bad output tensor")
            return out, out.data_ptr(), _ld(out.stride(), rows, cols)

        def activation_code(name):
            code = ACTIVATIONS.get(name)
            if code is None:
                raise ValueError(f"activations are {', '.join(ACTIVATIONS)}")
            return code

        def checked(out_dtype, default, fns):
            out_dtype = out_dtype or default
            if out_dtype not in fns:
                raise TypeError("results are bfloat16 or float32")
            return out_dtype

        current, device_of = torch._C._cuda_getDevice, torch.cuda.device

        def call(dev, fn, *args):
            if current() == dev:
                rc = fn(*args, raw_stream(dev))
            else:                                           # the entry points work on the current device
                with device_of(dev):
                    rc = fn(*args, raw_stream(dev))
            if rc != ok:
                raise _b.GemmError(rc)

        def gated(X, Wg, Wu, activation, keep, out):
            act = activation_code(activation)
            M, K = matrix(X)
            N = matrix(Wg)[0]
            dev = X.get_device()
            H, h, ldh = result(out, M, N, bf16, X)
            if keep:
                G, U = empty(M, N, dtype=bf16, device=X.device), empty(M, N, dtype=bf16, device=X.device)
                kept = (G.data_ptr(), N or 1, U.data_ptr(), N or 1)
            else:
                kept = (None, 0, None, 0)
            call(dev, f_gated, M, N, K, *operand(X, M, K, dev), *operand(Wg, N, K, dev), *operand(Wu, N, K, dev), act, h, ldh, *kept)
            return (H, G, U) if keep else H

        def grad(dY, Wd, G, U, activation):
            act = activation_code(activation)
            M, K = matrix(dY)
            N = matrix(Wd)[1]
            dev = dY.get_device()
            outs = [empty(M, N, dtype=bf16, device=dY.device) for _ in range(3)]
            places = [v for o in outs for v in (o.data_ptr(), N or 1)]
            call(dev, f_grad, M, N, K, *operand(dY, M, K, dev), *operand(Wd, K, N, dev), *operand(G, M, N, dev), *operand(U, M, N, dev), act,
                 *places)
            return tuple(outs)

        def bwd(dH, G, U, activation):
            act = activation_code(activation)
            M, N = matrix(dH)
            dev = dH.get_device()
            dG, dU = empty(M, N, dtype=bf16, device=dH.device), empty(M, N, dtype=bf16, device=dH.device)
            call(dev, fns["ffn_gated_bwd_bf16"], M, N, *operand(dH, M, N, dev), *operand(G, M, N, dev), *operand(U, M, N, dev), act,
                 dG.data_ptr(), N or 1, dU.data_ptr(), N or 1)
            return dG, dU

        def input_gradient(dG, Wg, dU, Wu, out, out_dtype):
            M, K = matrix(dG)
            N = matrix(Wg)[1]
            dev = dG.get_device()
            dtype = checked(out_dtype if out is None else out.dtype, bf16, dx)
            dX, p, ld = result(out, M, N, dtype, dG)
            call(dev, dx[dtype], M, N, K, *operand(dG, M, K, dev), *operand(Wg, K, N, dev), *operand(dU, M, K, dev), *operand(Wu, K, N, dev), p, ld)
            return dX

        def both_dw(dG, dU, X, out_dtype):
            K, M = matrix(dG)
            N = matrix(X)[1]
            dev = dG.get_device()
            dtype = checked(out_dtype, f32, dw2)
            dWg, dWu = empty(M, N, dtype=dtype, device=dG.device), empty(M, N, dtype=dtype, device=dG.device)
            call(dev, dw2[dtype], M, N, K, *operand(dG, K, M, dev), *operand(dU, K, M, dev), *operand(X, K, N, dev), dWg.data_ptr(), N or 1,
                 dWu.data_ptr(), N or 1)
            return dWg, dWu

        def one_dw(dY, X, out, out_dtype):
            K, M = matrix(dY)
            N = matrix(X)[1]
            dev = dY.get_device()
            dtype = checked(out_dtype if out is None else out.dtype, f32, dw1)
            dW, p, ld = result(out, M, N, dtype, dY)
            call(dev, dw1[dtype], M, N, K, *operand(dY, K, M, dev), *operand(X, K, N, dev), p, ld)
            return dW

        self.gated, self.grad, self.bwd, self.input_gradient, self.both_dw, self.one_dw = gated, grad, bwd, input_gradient, both_dw, one_dw


_helpers = None


def _h():
    global _helpers
    if _helpers is None:
        _helpers = _Helpers()
    return _helpers


def gated_linear(X, Wg, Wu, activation="silu", keep=False, out=None):
    """H = act(X . Wg^T) * (X . Wu^T): X M x K, Wg and Wu N x K, H M x N.  With ``keep`` (H, G, U): G = X . Wg^T and
    U = X . Wu^T in bf16, for ``gated_linear_grad``."""
    return (_helpers or _h()).gated(X, Wg, Wu, activation, keep, out)


def gated_linear_grad(dY, Wd, G, U, activation="silu"):
    """(dG, dU, H) of a block's output gradient dY (M x K), its down projection Wd (K x N) and what the forward
    pass kept: dG = (dY . Wd) * U * act'(G), dU = (dY . Wd) * act(G), H = act(G) * U."""
    return (_helpers or _h()).grad(dY, Wd, G, U, activation)


def gated_linear_bwd(dH, G, U, activation="silu"):
    """(dG, dU) of the gradient dH of H itself and what the forward pass kept: dG = dH * U * act'(G), dU = dH * act(G)."""
    return (_helpers or _h()).bwd(dH, G, U, activation)


def gated_linear_dx(dG, Wg, dU, Wu, out=None, out_dtype=None):
    """dG . Wg + dU . Wu (M x N, bf16 unless out_dtype or out says float32): dG, dU M x K, Wg, Wu K x N."""
    return (_helpers or _h()).input_gradient(dG, Wg, dU, Wu, out, out_dtype)


def gated_linear_dw(dG, dU, X, out_dtype=None):
    """(dG^T . X, dU^T . X), fp32 unless out_dtype says bfloat16: dG, dU tokens x M, X tokens x N."""
    return (_helpers or _h()).both_dw(dG, dU, X, out_dtype)


def linear_dw(dY, X, out=None, out_dtype=None):
    """dY^T . X, fp32 unless out_dtype or out says bfloat16: the weight gradient of a projection, dY tokens x M,
    X tokens x N."""
    return (_helpers or _h()).one_dw(dY, X, out, out_dtype)


def __getattr__(name):
    # The modules, which need torch at their definition.
    if name in ("GatedLinear", "GatedFeedForward"):
        from . import feedforward
        return getattr(feedforward, name)
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
