"""The gated feed-forward block and the adapters of many requests, the operators whose speed is followed.

A gated feed-forward block with weights Wg, Wu (N x K) and Wd (out x N) is y = H Wd^T with
H = act(X Wg^T) * (X Wu^T).  Its operators:

* "gated": H over X (M x K); with `keep` also G = X Wg^T and U = X Wu^T for the backward pass;
* "grad":  the gradients of G and U, and H again, from dY (M x K) and Wd (K x N):
  dH = dY . Wd, dG = dH * U * act'(G), dU = dH * act(G), H = act(G) * U;
* "dx":    dX = dG . Wg + dU . Wu, dG and dU M x K, Wg and Wu K x N;
* "dw":    dWg = dG^T . X and dWu = dU^T . X, dG and dU K tokens x M, X K tokens x N.

A projection W (out x in) that requests share, beside n adapters of rank r, A (n x r x in), B (n x out x r) and
a scale each; token t has adapter i(t), or none where i(t) is negative:

* "adapt":    y = x W^T + s_i (x A_i^T) B_i^T                     (x M x K, W N x K);
* "adapt_dx": dx = dy W + s_i (dy B_i) A_i                        (dy M x K, W K x N);
* "adapt_dw": dA_i = sum_t dh_t^T x_t and dB_i = sum_t dy_t^T h_t over the tokens of adapter i, from
  h_t = s_i x_t A_i^T and dh_t = s_i dy_t B_i as the two above leave them (x M x K, dy M x N).
"""
import math

import torch

own = False     # False: the plain form; True: the framework's kernels

_OUT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _ffn(name, op, M, N, K, act="silu", out="bf16", keep=False, pad=0):
    """out: the results' type.  pad: extra elements in each row of X's (dY's, dG's) buffer: a slice of a
    wider one."""
    c = {"op": op, "M": M, "N": N, "K": K, "act": act, "out": out, "keep": keep, "pad": pad}
    return {"name": name, **c} if name else c


def _adapt(name, op, M, N, K, n, r, q, mixed=False, bare=False, out="bf16", pad=0):
    """n adapters of rank r are held; the batch has q requests of M tokens in all (as many as there are adapters
    at most, each with one of its own).  mixed: the requests' tokens in no order.  bare: the last request has
    no adapter."""
    c = {"op": op, "M": M, "N": N, "K": K, "n": n, "r": r, "q": q, "mixed": mixed, "bare": bare, "out": out, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # One token through both projections of a feed-forward block: a read of the two weights.
        _ffn("gated_decode_m1", "gated", 1, 14336, 4096),
        # A batch of no particular size through a block with odd sizes.
        _ffn("gated_odd_m37", "gated", 37, 2051, 2049, "gelu"),
        # 2048 tokens in training: what the backward pass needs is kept.
        _ffn("gated_train", "gated", 2048, 11008, 4096, "silu", keep=True),
        # Gradients of the two products' results, 2048 tokens.
        _ffn("grad_train", "grad", 2048, 11008, 4096, "silu"),
        # A short fine-tuning batch, its gradient a slice of a wider one.
        _ffn("dx_short", "dx", 96, 4096, 11008, pad=64),
        # Input gradient of 2048 tokens.
        _ffn("dx_train", "dx", 2048, 4096, 11008),
        # Both weight gradients, fp32 for the optimiser.
        _ffn("dw_train", "dw", 11008, 4096, 2048, out="f32"),
        # A decode step of 16 requests, each with an adapter of its own.
        _adapt("adapt_decode_m16", "adapt", 16, 4096, 14336, 32, 16, 16),
        # A few tokens of three requests with odd sizes, one of them without an adapter.
        _adapt("adapt_odd_m37", "adapt", 37, 2051, 2049, 5, 7, 3, mixed=True, bare=True, out="f32"),
        # The prompts of five requests, one after the other.
        _adapt("adapt_prefill", "adapt", 2048, 4096, 4096, 16, 64, 5),
        # Adapters trained together: input gradient of eight jobs' tokens ...
        _adapt("adapt_dx_train", "adapt_dx", 2048, 4096, 11008, 8, 16, 8),
        # ... and every adapter's weight gradients.
        _adapt("adapt_dw_train", "adapt_dw", 2048, 11008, 4096, 8, 16, 8, out="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gated", "gated", "grad", "dx", "dw", "adapt", "adapt", "adapt_dx", "adapt_dw"])
    odd = rng.random() < 0.4
    tokens = _log_int(rng, 1, 4096)
    wide, deep = _log_int(rng, 1024, 14336), _log_int(rng, 1024, 14336)
    if op == "dw":          # both weights' rows, the model's width, the tokens
        M, N, K = wide, deep, tokens
    else:
        M, N, K = tokens, wide, deep
    if odd:
        N, K = N | 1, K | 1
        M = M | 1 if op == "dw" else M
    else:                   # sizes as most networks have them; a token count is any number
        N = N // 64 * 64
        M, K = (M // 64 * 64, K) if op == "dw" else (M, K // 64 * 64)
    most = 2048 * 11008 * 4096
    if M * N * K > most:    # fewer tokens
        if op == "dw":
            K = max(1, most // (M * N))
        else:
            M = max(1, most // (N * K))
    pad = rng.choice([0, 0, 64])
    if op in ("gated", "grad", "dx", "dw"):
        out = rng.choice(["bf16", "f32"]) if op in ("dx", "dw") else "bf16"
        return _ffn(None, op, M, N, K, rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), out,
                    op == "gated" and rng.random() < 0.5, pad)
    n = _log_int(rng, 1, 64)
    r = rng.choice([4, 8, 16, 16, 32, 64, 128, _log_int(rng, 1, 128)])
    q = _log_int(rng, 1, min(n, M)) if rng.random() < 0.5 else min(n, M)
    if op == "adapt_dw":    # the gradients of every adapter, and no product with W
        M = min(tokens, 2048)
        q = min(q, M)
    return _adapt(None, op, M, N, K, n, r, q, rng.random() < 0.3, q > 1 and rng.random() < 0.3,
                  rng.choice(["bf16", "f32"]), pad)


# ---- inputs -------------------------------------------------------------------------------------

def _activation(gen, rows, cols, pad=0, scale=1.0):
    """Some channels several times larger than others, as activations and their gradients have them."""
    dev = gen.device
    x = torch.randn(rows, cols + pad, device=dev, generator=gen) * scale
    x *= torch.exp(0.7 * torch.randn(cols + pad, device=dev, generator=gen))
    return x.to(torch.bfloat16)[:, :cols]


def _weight(gen, *shape):
    """A layer's weight: a unit input gives outputs of unit size."""
    return (torch.randn(*shape, device=gen.device, generator=gen) * 0.02).to(torch.bfloat16)


def _index(gen, case):
    """Each token's adapter (int32), -1 for none: q requests of random lengths, one token at least."""
    M, n, q = case["M"], case["n"], case["q"]
    dev = gen.device
    cuts = torch.sort(torch.randperm(M - 1, device=dev, generator=gen)[:q - 1] + 1).values if q > 1 else \
        torch.empty(0, dtype=torch.int64, device=dev)
    request = torch.bucketize(torch.arange(M, device=dev), cuts, right=True)
    adapter = torch.randperm(n, device=dev, generator=gen)[:q]
    if case["bare"]:
        adapter[q - 1] = -1
    index = adapter[request]
    if case["mixed"]:
        index = index[torch.randperm(M, device=dev, generator=gen)]
    return index.to(torch.int32)


def prepare(case, seed):
    op, M, N, K, pad = case["op"], case["M"], case["N"], case["K"], case["pad"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if op == "gated":
        s["X"], s["Wg"], s["Wu"] = _activation(gen, M, K, pad), _weight(gen, N, K), _weight(gen, N, K)
    elif op == "grad":
        s["dY"], s["Wd"] = _activation(gen, M, K, pad), _weight(gen, K, N)
        s["G"], s["U"] = _activation(gen, M, N), _activation(gen, M, N)
    elif op == "dx":
        s["dG"], s["dU"] = _activation(gen, M, K, pad), _activation(gen, M, K, pad)
        s["Wg"], s["Wu"] = _weight(gen, K, N), _weight(gen, K, N)
    elif op == "dw":
        s["dG"], s["dU"], s["X"] = _activation(gen, K, M, pad), _activation(gen, K, M, pad), _activation(gen, K, N)
    else:
        n, r = case["n"], case["r"]
        s["index"] = _index(gen, case)
        s["scale"] = torch.rand(n, device="cuda", generator=gen) + 0.5
        wide, narrow = (N, K) if op != "adapt_dx" else (K, N)       # the projection's outputs and inputs
        if op == "adapt_dw":
            s["x"], s["dy"] = _activation(gen, M, K, pad), _activation(gen, M, N)
            s["h"], s["dh"] = (torch.randn(M, r, device="cuda", generator=gen) for _ in range(2))
        else:
            s["x"] = _activation(gen, M, K, pad)
            s["W"] = _weight(gen, wide, narrow)
            s["A"], s["B"] = _weight(gen, n, r, narrow), _weight(gen, n, wide, r)
    return s


# ---- the pass -----------------------------------------------------------------------------------

def _act(name, g):
    """act(g) and act'(g)."""
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu":
        p = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    return torch.where(g > 0, g, 0.0), (g > 0).to(g.dtype)


def _spread(h, index, n):
    """h (M x r) in its adapter's columns of an M x (n r) matrix, zeros elsewhere."""
    pick = (index[:, None] == torch.arange(n, device=h.device)).to(h.dtype)
    return (pick[:, :, None] * h[:, None, :]).flatten(1)


def _own(s, out):
    from paper_2512_13282_amd import binding as b
    case = s["case"]
    op = case["op"]
    if op == "gated":
        return b.gated_linear(s["X"], s["Wg"], s["Wu"], case["act"], keep=case["keep"])
    if op == "grad":
        return b.gated_linear_grad(s["dY"], s["Wd"], s["G"], s["U"], case["act"])
    if op == "dx":
        return b.gated_linear_dx(s["dG"], s["Wg"], s["dU"], s["Wu"], out_dtype=out)
    if op == "dw":
        return b.gated_linear_dw(s["dG"], s["dU"], s["X"], out_dtype=out)
    if op == "adapt_dw":
        return b.linear_adapters_dw(s["x"], s["dy"], s["h"], s["dh"], s["index"], case["n"], out_dtype=out)
    adapters = b.Adapters(s["A"], s["B"], s["scale"])
    if op == "adapt":
        return b.linear_adapters(s["x"], s["W"], adapters, s["index"], out_dtype=out)
    return b.linear_adapters_dx(s["x"], s["W"], adapters, s["index"], out_dtype=out)


def run(state):
    s, case = state, state["case"]
    op, out = case["op"], _OUT[case["out"]]
    if own:
        return _own(s, out)
    if op == "gated":
        x = s["X"].float()
        g, u = x @ s["Wg"].float().t(), x @ s["Wu"].float().t()
        h = (_act(case["act"], g)[0] * u).to(out)
        return (h, g.to(out), u.to(out)) if case["keep"] else h
    if op == "grad":
        dh, u = s["dY"].float() @ s["Wd"].float(), s["U"].float()
        a, da = _act(case["act"], s["G"].float())
        return (dh * u * da).to(out), (dh * a).to(out), (a * u).to(out)
    if op == "dx":
        return (s["dG"].float() @ s["Wg"].float() + s["dU"].float() @ s["Wu"].float()).to(out)
    if op == "dw":
        x = s["X"].float()
        return (s["dG"].float().t() @ x).to(out), (s["dU"].float().t() @ x).to(out)
    n, r, index = case["n"], case["r"], s["index"]
    if op == "adapt_dw":
        dA = _spread(s["dh"], index, n).t() @ s["x"].float()
        dB = _spread(s["h"], index, n).t() @ s["dy"].float()
        return dA.view(n, r, -1).to(out), dB.view(n, r, -1).transpose(1, 2).to(out).contiguous()
    x, W, A, B = (s[k].float() for k in ("x", "W", "A", "B"))
    row = torch.arange(len(index), device=index.device)
    held = index.clamp(min=0).long()
    scale = s["scale"][held][:, None]
    if op == "adapt":
        h = (x @ A.flatten(0, 1).t()).view(-1, n, r)[row, held] * scale
        return (x @ W.t() + _spread(h, index, n) @ B.transpose(1, 2).reshape(n * r, -1)).to(out)
    dh = (x @ B.transpose(0, 1).reshape(-1, n * r)).view(-1, n, r)[row, held] * scale
    return (x @ W + _spread(dh, index, n) @ A.flatten(0, 1)).to(out)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    op, M, N, K = case["op"], case["M"], case["N"], case["K"]
    o = _OUT[case["out"]].itemsize
    if op == "gated":
        return {"bytes": 2 * M * K + 4 * N * K + (6 if case["keep"] else 2) * M * N, "flops": 4 * M * N * K}
    if op == "grad":
        return {"bytes": 2 * M * K + 2 * N * K + 10 * M * N, "flops": 2 * M * N * K}
    if op == "dx":
        return {"bytes": 4 * M * K + 4 * N * K + o * M * N, "flops": 4 * M * N * K}
    if op == "dw":
        return {"bytes": 4 * M * K + 2 * N * K + 2 * o * M * N, "flops": 4 * M * N * K}
    n, r = case["n"], case["r"]
    used = case["q"] - (1 if case["bare"] else 0)
    if op == "adapt_dw":
        return {"bytes": 2 * M * (N + K) + 8 * M * r + 4 * M + o * n * r * (N + K), "flops": 2 * M * r * (N + K)}
    return {"bytes": 2 * M * K + 2 * N * K + o * M * N + 2 * used * r * (N + K) + 4 * M,
            "flops": 2 * M * N * K + 2 * M * r * (N + K)}


# ---- the definitions in 64 bits -----------------------------------------------------------------

def _exact_act(name, g):
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * torch.sigmoid(-g)
    if name == "gelu":
        p = 0.5 * torch.special.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":         # (1 + tanh z) / 2 = sigmoid(2 z)
        z2 = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        p = torch.sigmoid(z2)
        return g * p, p + g * p * torch.sigmoid(-z2) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * g ** 2)
    return g.clamp(min=0), torch.sign(g).clamp(min=0)


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    d = {k: v.double().contiguous() for k, v in s.items() if torch.is_tensor(v) and k != "index"}
    if op == "gated":
        g = torch.mm(d["X"], d["Wg"].t().contiguous())
        u = torch.mm(d["X"], d["Wu"].t().contiguous())
        h = _exact_act(case["act"], g)[0] * u
        return (h, g, u) if case["keep"] else h
    if op == "grad":
        a, da = _exact_act(case["act"], d["G"])
        dh = torch.mm(d["dY"], d["Wd"])
        return dh * d["U"] * da, dh * a, a * d["U"]
    if op == "dx":
        return torch.mm(torch.cat((d["dG"], d["dU"]), 1), torch.cat((d["Wg"], d["Wu"]), 0))
    if op == "dw":
        both = torch.mm(torch.cat((d["dG"], d["dU"]), 1).t().contiguous(), d["X"])
        return both[:case["M"]], both[case["M"]:]
    n, r = case["n"], case["r"]
    which = s["index"].cpu().tolist()
    rows = {i: torch.tensor([t for t, j in enumerate(which) if j == i], dtype=torch.int64, device="cuda") for i in set(which) if i >= 0}
    if op == "adapt_dw":
        dA = torch.zeros(n, r, case["K"], dtype=torch.float64, device="cuda")
        dB = torch.zeros(n, case["N"], r, dtype=torch.float64, device="cuda")
        for i, t in rows.items():
            dA[i] = torch.mm(d["dh"][t].t().contiguous(), d["x"][t])
            dB[i] = torch.mm(d["dy"][t].t().contiguous(), d["h"][t])
        return dA, dB
    y = torch.mm(d["x"], d["W"].t().contiguous() if op == "adapt" else d["W"])
    for i, t in rows.items():
        down, up = (d["A"][i].t(), d["B"][i].t()) if op == "adapt" else (d["B"][i], d["A"][i])
        y[t] += torch.mm(torch.mm(d["x"][t], down.contiguous()), up.contiguous()) * d["scale"][i]
    return y
