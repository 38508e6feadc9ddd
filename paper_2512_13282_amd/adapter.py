"""A linear layer whose weight is frozen in 4 bits, with a trainable low-rank adapter: the
block-scaled operators together, as fine-tuning and then decoding use them.

    y = x W^T + (x A^T) B^T        W: 4-bit (n_out x n_in), A: rank x n_in, B: n_out x rank

The forward pass keeps x and x A^T for the backward pass in 8 bits, half of what bf16 takes; the
backward pass takes the adapter's gradients from what it kept and the input's from the packed
weight.  ``python -m paper_2512_13282_amd.adapter`` trains a layer towards another one on
synthetic data and then decodes a token through it.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad

from . import binding


def differentiated(*tensors) -> bool:
    """Whether a call on these tensors may be asked for derivatives: it then takes its autograd function, which gives
    gradients and refuses forward-mode tangents, where the helpers alone would drop them."""
    return torch.is_grad_enabled() or any(forward_ad.unpack_dual(t).tangent is not None for t in tensors)


class _FirstDerivative(torch.autograd.Function):
    """A gradient that came out of kernels which autograd does not see, as a function of the tensors behind it:
    whoever differentiates it again is told so, instead of taking it for a constant."""

    @staticmethod
    def forward(ctx, gradient, *behind):
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("AdapterLinear has first derivatives only")


class _AdapterLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, A, B):
        h = binding.mm_bf16_f32(x, A.t()).to(torch.bfloat16)                 # tokens x rank
        y = binding.linear_mx4(x, W, out_dtype=torch.float32)
        y += binding.mm_bf16_f32(h, B.t())
        X, H = binding.pack_mx8(x), binding.pack_mx8(h)
        ctx.save_for_backward(X.codes, X.scales, H.codes, H.scales, A, B)
        ctx.W, ctx.cols = W, (X.cols, H.cols)
        return y.to(torch.bfloat16)

    @staticmethod
    def backward(ctx, dy):
        xc, xs, hc, hs, A, B = ctx.saved_tensors
        X, H = binding.MxMatrix(xc, xs, ctx.cols[0]), binding.MxMatrix(hc, hs, ctx.cols[1])
        dy = dy.contiguous()
        dh = binding.mm_bf16_f32(dy, B).to(torch.bfloat16)                   # dy . B
        dB = binding.linear_mx8_dw(dy, H, out_dtype=torch.bfloat16)          # dy^T . h
        dA = binding.linear_mx8_dw(dh, X, out_dtype=torch.bfloat16)          # dh^T . x
        dx = None
        if ctx.needs_input_grad[0]:
            dx = binding.linear_mx4_dx(dy, ctx.W, out_dtype=torch.float32)   # dy . W
            dx += binding.mm_bf16_f32(dh, A)
            dx = dx.to(torch.bfloat16)
        if torch.is_grad_enabled():                                          # create_graph=True
            dx, dA, dB = (None if g is None else _FirstDerivative.apply(g, dy, A, B) for g in (dx, dA, dB))
        return dx, None, dA, dB


def _rows16(codes):
    """Codes with their rows a multiple of 16 bytes apart, as packing lays them out: where they are not
    (a module that is moved or loaded gets them one after the other), every product would copy them."""
    rows, width = codes.shape
    if rows < 2 or codes.stride(0) % 16 == 0 and codes.stride(1) == 1:
        return codes
    out = torch.empty_strided((rows, width), (-(-width // 16) * 16, 1), dtype=codes.dtype, device=codes.device)
    return out.copy_(codes)


class AdapterLinear(torch.nn.Module):
    """``weight``: a bf16 matrix (n_out x n_in) on the GPU, packed to 4 bits here, or an ``MxMatrix``.  Its parts are
    buffers of the module, so that the adapter is saved, loaded and moved with the weight it was trained over."""

    def __init__(self, weight, rank: int):
        super().__init__()
        codes, scales, n_in = weight if isinstance(weight, binding.MxMatrix) else binding.pack_mx4(weight)
        n_out, dev = codes.shape[0], codes.device
        self.register_buffer("weight_codes", _rows16(codes))
        self.register_buffer("weight_scales", scales)
        self.A = torch.nn.Parameter((torch.randn(rank, n_in, device=dev) / n_in ** 0.5).to(torch.bfloat16))
        self.B = torch.nn.Parameter(torch.zeros(n_out, rank, device=dev, dtype=torch.bfloat16))

    @property
    def weight(self) -> binding.MxMatrix:
        return binding.MxMatrix(self.weight_codes, self.weight_scales, self.A.shape[1])

    @weight.setter
    def weight(self, W: binding.MxMatrix):
        self.weight_codes, self.weight_scales = _rows16(W.codes), W.scales

    def _apply(self, fn, *args, **kwargs):
        super()._apply(fn, *args, **kwargs)
        self.weight_codes = _rows16(self.weight_codes)
        return self

    def forward(self, x):
        """x: tokens x n_in, bf16 (one token to a batch of prompts).  First derivatives only: a gradient of a
        gradient raises, and so does a forward-mode tangent."""
        if differentiated(x, self.A, self.B):
            return _AdapterLinear.apply(x, self.weight, self.A, self.B)
        h = binding.mm_bf16_f32(x, self.A.t()).to(torch.bfloat16)
        y = binding.linear_mx4(x, self.weight, out_dtype=torch.float32)
        y += binding.mm_bf16_f32(h, self.B.t())
        return y.to(torch.bfloat16)


def train(steps: int = 30, n_in: int = 512, n_out: int = 384, rank: int = 16, tokens: int = 256, seed: int = 0):
    """Fits the adapter of a packed layer to a layer that differs from it by a low-rank matrix.
    Returns (layer, the losses)."""
    torch.manual_seed(seed)
    dev = torch.device("cuda")
    W = (torch.randn(n_out, n_in, device=dev) / n_in ** 0.5).to(torch.bfloat16)
    layer = AdapterLinear(W, rank)
    base = binding.unpack_mx(layer.weight).float()
    target = base + 0.5 * (torch.randn(n_out, 4, device=dev) @ torch.randn(4, n_in, device=dev)) / n_in ** 0.5
    opt = torch.optim.Adam(layer.parameters(), lr=2e-2)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, n_in, device=dev).to(torch.bfloat16)
        loss = ((layer(x).float() - x.float() @ target.t()) ** 2).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    return layer, losses


if __name__ == "__main__":
    layer, losses = train()
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    with torch.no_grad():
        token = torch.randn(1, layer.weight.cols, device="cuda").to(torch.bfloat16)
        print("decoded token:", tuple(layer(token).shape), layer(token).dtype)
