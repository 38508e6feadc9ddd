"""The gated feed-forward block and the projection with adapters in 64 bits, with bounds on what their kernels'
roundings can add (plain torch, on whatever device the operands are).

Bounds.  A product's fp32 sum of K exact terms is off by at most K steps of 2^-23 of the sum of the terms' magnitudes
(every addition, whichever way it rounds, by a step of a partial sum).  A result in bf16 adds half a step, 2^-8 of it.
"""
import math

import torch

STEP = 2.0 ** -23
ACTIVATIONS = ("silu", "gelu", "gelu_tanh", "relu")
# act is off by at most 2^-20 (1 + |act|) and act' by 2^-19: the hardware's 2^x and 1 / x are good to 2^-22, the exponent's
# argument is off by |z| 2^-23, and |z| p (1 - p), z^2 p (1 - p) stay below 0.6.
ACT_ERROR, SLOPE_ERROR = 2.0 ** -20, 2.0 ** -19


def act(name, g):
    """act(g), act'(g) in 64 bits."""
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * torch.sigmoid(-g))
    if name == "gelu":
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        p = torch.sigmoid(c * (g + 0.044715 * g ** 3))
        return g * p, p + g * p * (1 - p) * c * (1 + 3 * 0.044715 * g * g)
    return torch.clamp(g, min=0), (g > 0).to(g.dtype)


def product(a, b):
    """(a . b, its bound) in 64 bits."""
    a, b = a.double().contiguous(), b.double().contiguous()
    return a @ b, (a.abs() @ b.abs()) * (a.shape[1] * STEP)


def rounded(value, bound, dtype):
    """The bound of a result that is stored as `dtype`."""
    half = torch.finfo(dtype).eps / 2 if dtype == torch.bfloat16 else 0.0
    return bound + half * (value.abs() + bound) + 1e-37


def gated(x, wg, wu, name):
    """((H, bound), (G, bound), (U, bound)), all stored in bf16."""
    g, eg = product(x, wg.t())
    u, eu = product(x, wu.t())
    a, _ = act(name, g)
    ea = 1.2 * eg + ACT_ERROR * (1 + a.abs())                # |act'| stays below 1.2
    eh = ea * (u.abs() + eu) + a.abs() * eu + 2.0 ** -23 * (a * u).abs()
    return [(v, rounded(v, e, torch.bfloat16)) for v, e in ((a * u, eh), (g, eg), (u, eu))]


def grad(dy, wd, g, u, name):
    """((dG, bound), (dU, bound), (H, bound))."""
    d, ed = product(dy, wd)
    g, u = g.double(), u.double()
    a, s = act(name, g)
    ea, es = ACT_ERROR * (1 + a.abs()), SLOPE_ERROR * (1 + s.abs())
    out = []
    for v, e in ((d * u * s, ed * (u * s).abs() + (d.abs() + ed) * u.abs() * es),
                 (d * a, ed * a.abs() + (d.abs() + ed) * ea), (a * u, ea * u.abs())):
        out.append((v, rounded(v, e + 2.0 ** -22 * v.abs(), torch.bfloat16)))
    return out


def dx(dg, wg, du, wu, dtype):
    v, e = product(torch.cat((dg, du), 1), torch.cat((wg, wu), 0))
    return v, rounded(v, e, dtype)


def dw(dy, x, dtype):
    v, e = product(dy.t(), x)
    return v, rounded(v, e, dtype)


def tokens_of(index, n):
    """Each adapter's tokens."""
    which = index.tolist()
    return [[t for t, j in enumerate(which) if j == i] for i in range(n)]


def adapted(x, w, down, up, scale, index, dtype):
    """((y, bound), (h, bound)): y = x . w plus, for the tokens of adapter i, h . up[i] with h = s_i x . down[i]
    (w K x N, down n x K x r, up n x r x N).  h is in fp32; the second product leaves 2^-16 of it out where y is
    bf16, and takes it in three parts, each a term of its own."""
    y, e = product(x, w)
    n, r = down.shape[0], down.shape[2]
    h = torch.zeros(x.shape[0], r, dtype=torch.float64, device=x.device)
    eh = torch.zeros_like(h)
    for i, t in enumerate(tokens_of(index, n)):
        if not t:
            continue
        s = float(scale[i]) if scale is not None else 1.0
        v, ev = product(x[t], down[i])
        h[t], eh[t] = v * s, (ev + 2.0 ** -23 * v.abs()) * abs(s)
        b = up[i].double()
        y[t] += h[t] @ b
        left = 2.0 ** -16 if dtype == torch.bfloat16 else 0.0
        e[t] += eh[t] @ b.abs() + (h[t].abs() @ b.abs()) * (left + (3 * r + 4) * STEP)
    e += 4 * STEP * y.abs()
    return (y, rounded(y, e, dtype)), (h, eh + 8 * STEP * h.abs() + 1e-37)      # up to 8 planes of h


def adapter_dw(x, dy, h, dh, index, n, dtype):
    """((dA, bound), (dB, bound)): h and dh in three bf16 parts, two (2^-16 left out) where the results are bf16."""
    M, K = x.shape
    N, r = dy.shape[1], h.shape[1]
    out = []
    for z, p, cols in ((x, dh, K), (dy, h, N)):
        v = torch.zeros(n, r, cols, dtype=torch.float64, device=x.device)
        e = torch.zeros_like(v)
        for i, t in enumerate(tokens_of(index, n)):
            if t:
                q, zz = p[t].double().t().contiguous(), z[t].double()
                v[i] = q @ zz
                e[i] = (q.abs() @ zz.abs()) * ((2.0 ** -16 if dtype == torch.bfloat16 else 0.0) + (3 * len(t) + 4) * STEP)
        out.append((v, rounded(v, e, dtype)))
    (da, ea), (db, eb) = out
    return (da, ea), (db.transpose(1, 2), eb.transpose(1, 2))


def assert_within(got, want, what=""):
    value, bound = want
    off = (got.double() - value).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} past the bound, first at {i}: got {got[i].item()}, "
                             f"want {value[i].item()} within {bound[i].item()}")
