"""The gated feed-forward block and a projection with adapters as torch modules: the operators of ffn.py and adapters.py
behind autograd, as training and then decoding use them.

    GatedLinear:        h = act(x Wg^T) * (x Wu^T)
    GatedFeedForward:   y = h Wd^T, its backward pass without dH in memory
    AdaptersLinear:     y = x W^T + s_i (x A_i^T) B_i^T, token t of adapter i = index[t]

The forward pass keeps G = x Wg^T and U = x Wu^T in bf16 for the backward pass, which forms h again from them.
Inputs are matrices of tokens x n_in in bf16; gradients are first derivatives; a gradient of a gradient raises, and so does a
forward-mode tangent.
``python -m paper_2512_13282_amd.feedforward`` trains a block whose down projection has adapters of several jobs, on
synthetic data, and then decodes a token of each.
"""
from __future__ import annotations

import torch

from . import binding
from .adapter import differentiated
from .mx import _ld


class _FirstDerivative(torch.autograd.Function):
    """A gradient that came out of kernels which autograd does not see, as a function of the tensors behind it:
    whoever differentiates it again is told so, instead of taking it for a constant."""

    @staticmethod
    def forward(ctx, gradient, *behind):
        return gradient.view_as(gradient)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the feed-forward and adapter operators have first derivatives only")


def _gradients(gradients, *behind):
    if torch.is_grad_enabled():                                              # create_graph=True
        return tuple(None if g is None else _FirstDerivative.apply(g, *behind) for g in gradients)
    return tuple(gradients)


def _linear(x, W):
    """x . W^T rounded once to bf16."""
    if x.dtype != torch.bfloat16 or W.dtype != torch.bfloat16:
        raise TypeError("expected bfloat16 operands")
    if x.dim() != 2 or W.dim() != 2 or W.shape[1] != x.shape[1]:
        raise ValueError("operand sizes do not fit")
    if not x.is_cuda or not W.is_cuda or x.get_device() != W.get_device():
        raise ValueError("operands must be on the same GPU")
    (M, K), N = x.shape, W.shape[0]
    y = torch.empty(M, N, dtype=torch.bfloat16, device=x.device)
    with torch.cuda.device(x.device):
        rc = binding.gemm_bf16_bf16_bt(M, N, K, x.data_ptr(), _ld(x.stride(), M, K), W.data_ptr(), _ld(W.stride(), N, K), y.data_ptr(), N or 1,
                                       torch.cuda.current_stream(x.device).cuda_stream)
    if rc != binding.GEMM_OK:
        raise binding.GemmError(rc)
    return y


class _GatedLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, Wg, Wu, activation):
        h, G, U = binding.gated_linear(x, Wg, Wu, activation, keep=True)
        ctx.save_for_backward(x, Wg, Wu, G, U)
        ctx.activation = activation
        return h

    @staticmethod
    def backward(ctx, dh):
        x, Wg, Wu, G, U = ctx.saved_tensors
        dG, dU = binding.gated_linear_bwd(dh.contiguous(), G, U, ctx.activation)
        dx = dWg = dWu = None
        if ctx.needs_input_grad[0]:
            dx = binding.gated_linear_dx(dG, Wg, dU, Wu)
        if ctx.needs_input_grad[1] or ctx.needs_input_grad[2]:
            dWg, dWu = binding.gated_linear_dw(dG, dU, x, out_dtype=torch.bfloat16)
        return *_gradients((dx, dWg, dWu), dh, x, Wg, Wu), None


class _GatedFeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, Wg, Wu, Wd, activation):
        h, G, U = binding.gated_linear(x, Wg, Wu, activation, keep=True)
        ctx.save_for_backward(x, Wg, Wu, Wd, G, U)
        ctx.activation = activation
        return _linear(h, Wd)

    @staticmethod
    def backward(ctx, dy):
        x, Wg, Wu, Wd, G, U = ctx.saved_tensors
        need = ctx.needs_input_grad
        given, dy = dy, dy.contiguous()
        dG, dU, h = binding.gated_linear_grad(dy, Wd, G, U, ctx.activation)
        dx = dWg = dWu = dWd = None
        if need[0]:
            dx = binding.gated_linear_dx(dG, Wg, dU, Wu)
        if need[1] or need[2]:
            dWg, dWu = binding.gated_linear_dw(dG, dU, x, out_dtype=torch.bfloat16)
        if need[3]:
            dWd = binding.linear_dw(dy, h, out_dtype=torch.bfloat16)
        return *_gradients((dx, dWg, dWu, dWd), given, x, Wg, Wu, Wd), None


class _AdaptersLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, A, B, scale, index):
        if ctx.needs_input_grad[4]:
            raise RuntimeError("the adapters' scales have no gradient")
        y, h = binding.linear_adapters(x, W, binding.Adapters(A, B, scale), index, keep=True)
        ctx.save_for_backward(x, W, A, B, scale, index, h)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, W, A, B, scale, index, h = ctx.saved_tensors
        need = ctx.needs_input_grad
        given, dy = dy, dy.contiguous()
        dx, dh = binding.linear_adapters_dx(dy, W, binding.Adapters(A, B, scale), index, keep=True)
        dW = dA = dB = None
        if need[1]:
            dW = binding.linear_dw(dy, x, out_dtype=torch.bfloat16)
        if need[2] or need[3]:
            dA, dB = binding.linear_adapters_dw(x, dy, h, dh, index, A.shape[0], out_dtype=torch.bfloat16)
        return *_gradients((dx, dW, dA, dB), given, x, W, A, B), None, None


def _weight(*shape, device):
    return torch.nn.Parameter((torch.randn(*shape, device=device) / shape[-1] ** 0.5).to(torch.bfloat16))


class GatedLinear(torch.nn.Module):
    """act(x Wg^T) * (x Wu^T), tokens x n_hidden, from bf16 parameters ``gate`` and ``up`` (n_hidden x n_in)."""

    def __init__(self, n_in: int, n_hidden: int, activation: str = "silu", device="cuda"):
        super().__init__()
        self.gate, self.up = _weight(n_hidden, n_in, device=device), _weight(n_hidden, n_in, device=device)
        self.activation = activation

    def forward(self, x):
        if differentiated(x, self.gate, self.up):
            return _GatedLinear.apply(x, self.gate, self.up, self.activation)
        return binding.gated_linear(x, self.gate, self.up, self.activation)


class GatedFeedForward(GatedLinear):
    """The block: ``GatedLinear`` and a down projection ``down`` (n_out x n_hidden)."""

    def __init__(self, n_in: int, n_hidden: int, n_out: int | None = None, activation: str = "silu", device="cuda"):
        super().__init__(n_in, n_hidden, activation, device)
        self.down = _weight(n_in if n_out is None else n_out, n_hidden, device=device)

    def forward(self, x):
        if differentiated(x, self.gate, self.up, self.down):
            return _GatedFeedForward.apply(x, self.gate, self.up, self.down, self.activation)
        return _linear(binding.gated_linear(x, self.gate, self.up, self.activation), self.down)


class AdaptersLinear(torch.nn.Module):
    """A projection ``weight`` (n_out x n_in bf16, a buffer that does not learn) with ``n`` trainable adapters of rank ``rank``.
    Its scales (a buffer) are fp32, stay so where the module is converted to another type, and have no
    gradient.  ``forward(x, index)``: index holds each token's adapter (int32), -1 for none."""

    def __init__(self, weight, n: int, rank: int, scale: float = 1.0):
        super().__init__()
        n_out, n_in = weight.shape
        self.register_buffer("weight", weight)
        self.register_buffer("scale", torch.full((n,), scale, device=weight.device, dtype=torch.float32))
        self.A = _weight(n, rank, n_in, device=weight.device)
        self.B = torch.nn.Parameter(torch.zeros(n, n_out, rank, device=weight.device, dtype=torch.bfloat16))

    def _apply(self, fn, *args, **kwargs):
        scale = self.scale
        super()._apply(fn, *args, **kwargs)
        if self.scale.dtype != torch.float32:       # a module that is converted keeps its fp32 scales
            self.scale = scale.to(self.scale.device)
        return self

    def forward(self, x, index):
        if differentiated(x, self.weight, self.A, self.B, self.scale):
            return _AdaptersLinear.apply(x, self.weight, self.A, self.B, self.scale, index)
        return binding.linear_adapters(x, self.weight, binding.Adapters(self.A, self.B, self.scale), index)


def train(steps: int = 20, n_in: int = 256, n_hidden: int = 512, jobs: int = 3, rank: int = 8, tokens: int = 192, seed: int = 0):
    """Trains the adapters of several jobs in one batch, on the down projection of a frozen block, towards a target of
    their own each.  Returns (the gated part, the projection, the losses)."""
    torch.manual_seed(seed)
    dev = torch.device("cuda")
    gated = GatedLinear(n_in, n_hidden).requires_grad_(False)
    down = AdaptersLinear((torch.randn(n_in, n_hidden, device=dev) / n_hidden ** 0.5).to(torch.bfloat16), jobs, rank)
    targets = torch.randn(jobs, n_in, device=dev)
    opt = torch.optim.Adam(down.parameters(), lr=1e-2)
    losses = []
    for _ in range(steps):
        x = torch.randn(tokens, n_in, device=dev).to(torch.bfloat16)
        index = torch.randint(0, jobs, (tokens,), device=dev, dtype=torch.int32)
        loss = ((down(gated(x), index).float() - targets[index.long()]) ** 2).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    return gated, down, losses


if __name__ == "__main__":
    gated, down, losses = train()
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
    with torch.no_grad():
        jobs = down.A.shape[0]
        x = torch.randn(jobs, gated.gate.shape[1], device="cuda").to(torch.bfloat16)
        y = down(gated(x), torch.arange(jobs, device="cuda", dtype=torch.int32))
        print("decoded a token of each job:", tuple(y.shape), y.dtype)
