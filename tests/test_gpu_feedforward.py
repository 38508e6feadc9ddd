"""The feed-forward and adapter modules: outputs and gradients against the formulas in 64 bits and against differences, in a
run of the operators together, in a captured training step, and on streams of their own."""
import pytest
import torch

import fused_reference as ref
from paper_2512_13282_amd import feedforward as ff
from test_gpu_ffn import BF16, DEV

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8       # a bf16 rounding


def close(got, want, size, roundings):
    """Within `roundings` bf16 roundings of the sum of the terms' magnitudes (fp32 sums are far below that)."""
    off = (got.double() - want).abs()
    assert torch.all(off <= roundings * HALF * size + 1e-30), (off / (HALF * size + 1e-30)).max().item()


def plain_block(x, wg, wu, wd, name):
    g, u = x @ wg.t(), x @ wu.t()
    h = ref.act(name, g)[0] * u
    return (h @ wd.t()) if wd is not None else h


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
@pytest.mark.parametrize("tokens,n_in,n_hidden,n_out", [(1, 64, 96, 32), (33, 96, 130, 72), (200, 515, 264, 130)])
def test_block_gradients(tokens, n_in, n_hidden, n_out, name):
    torch.manual_seed(tokens)
    block = ff.GatedFeedForward(n_in, n_hidden, n_out, name)
    x = torch.randn(tokens, n_in, device=DEV).to(BF16).requires_grad_()
    dy = torch.randn(tokens, n_out, device=DEV).to(BF16)
    y = block(x)
    y.backward(dy)
    X, wg, wu, wd = (t.detach().double() for t in (x, block.gate, block.up, block.down))
    d = dy.double()
    g, u = X @ wg.t(), X @ wu.t()
    a, s = ref.act(name, g)
    dh = d @ wd
    dg, du, h = dh * u * s, dh * a, a * u
    # Magnitudes, with what a rounded g or u moves: at most a rounding of g and of u each through act, act' and the products.
    G, U = X.abs() @ wg.abs().t(), X.abs() @ wu.abs().t()
    sh = (a.abs() + 1.2 * g.abs()) * u.abs()
    sdh = d.abs() @ wd.abs()
    sdg = sdh * u.abs() * (s.abs() + g.abs() + 1e-3)             # |act''| stays below 1.1; relu has a step where g is 0
    sdu = sdh * (a.abs() + 1.2 * g.abs())
    if name == "relu":
        assert G.min() >= 0
    for got, want, size, n in ((y.detach(), h @ wd.t(), sh @ wd.abs().t(), 3),
                               (x.grad, dg @ wg + du @ wu, sdg @ wg.abs() + sdu @ wu.abs(), 5),
                               (block.gate.grad, dg.t() @ X, sdg.t() @ X.abs(), 5), (block.up.grad, du.t() @ X, sdu.t() @ X.abs(), 5),
                               (block.down.grad, d.t() @ h, d.abs().t() @ sh, 4)):
        close(got, want, size, n)
    with torch.no_grad():
        assert torch.equal(block(x), y)


@pytest.mark.parametrize("tokens,n_in,n_hidden,n_out,n,rank", [(1, 64, 96, 32, 1, 4), (37, 96, 130, 72, 5, 7), (200, 520, 264, 136, 3, 16)])
def test_gated_part_with_adapters_after_it(tokens, n_in, n_hidden, n_out, n, rank):
    """The operators together: a gated product, then a down projection with each request's adapter."""
    torch.manual_seed(tokens)
    gated = ff.GatedLinear(n_in, n_hidden)
    down = ff.AdaptersLinear((torch.randn(n_out, n_hidden, device=DEV) / n_hidden ** 0.5).to(BF16), n, rank, scale=0.75)
    with torch.no_grad():
        down.B.copy_(torch.randn(n, n_out, rank, device=DEV) / rank ** 0.5)
    x = torch.randn(tokens, n_in, device=DEV).to(BF16).requires_grad_()
    index = torch.randint(-1, n, (tokens,), device=DEV, dtype=torch.int32)
    dy = torch.randn(tokens, n_out, device=DEV).to(BF16)
    y = down(gated(x), index)
    y.backward(dy)
    X, wg, wu, W, A, B = (t.detach().double() for t in (x, gated.gate, gated.up, down.weight, down.A, down.B))
    d, pick = dy.double(), (index[:, None] == torch.arange(n, device=DEV)).double()
    g, u = X @ wg.t(), X @ wu.t()
    a, s = ref.act("silu", g)
    h = a * u
    own = index.clamp(min=0).long()
    has = (index >= 0).double()[:, None]
    low = torch.einsum("tk,tjk->tj", h, A[own]) * 0.75 * has
    dlow = torch.einsum("tn,tnj->tj", d, B[own]) * 0.75 * has
    want = h @ W.t() + torch.einsum("tj,tnj->tn", low, B[own])
    dh = d @ W + torch.einsum("tj,tjk->tk", dlow, A[own])
    dg, du = dh * u * s, dh * a
    sh = (a.abs() + 1.2 * g.abs()) * u.abs()
    slow = torch.einsum("tk,tjk->tj", sh, A[own].abs())
    sdlow = torch.einsum("tn,tnj->tj", d.abs(), B[own].abs())
    sdh = d.abs() @ W.abs() + torch.einsum("tj,tjk->tk", sdlow, A[own].abs())
    sdg, sdu = sdh * u.abs() * (s.abs() + g.abs()), sdh * (a.abs() + 1.2 * g.abs())
    for got, value, size, k in (
            (y.detach(), want, sh @ W.abs().t() + torch.einsum("tj,tnj->tn", slow, B[own].abs()), 4),
            (x.grad, dg @ wg + du @ wu, sdg @ wg.abs() + sdu @ wu.abs(), 6),
            (gated.gate.grad, dg.t() @ X, sdg.t() @ X.abs(), 6), (gated.up.grad, du.t() @ X, sdu.t() @ X.abs(), 6),
            (down.A.grad, torch.einsum("ti,tj,tk->ijk", pick, dlow, h), torch.einsum("ti,tj,tk->ijk", pick, sdlow, sh), 4),
            (down.B.grad, torch.einsum("ti,tn,tj->inj", pick, d, low), torch.einsum("ti,tn,tj->inj", pick, d.abs(), slow), 4)):
        close(got, value, size, k)
    with torch.no_grad():
        assert torch.equal(down(gated(x), index), y)
        # One token at a time runs other kernels, plans and slices: fp32 sums in another order, rounded to bf16 twice.
        one = torch.cat([down(gated(x[i:i + 1]), index[i:i + 1]) for i in range(min(tokens, 5))])
        close(one, y[:5].double(), (sh @ W.abs().t() + torch.einsum("tj,tnj->tn", slow, B[own].abs()))[:5], 2)


def test_gradients_against_differences():
    """A directional derivative of the block in 64 bits against the gradients that the kernels give."""
    torch.manual_seed(5)
    block = ff.GatedFeedForward(64, 96, 40, "gelu")
    x = torch.randn(50, 64, device=DEV).to(BF16).requires_grad_()
    c = torch.randn(50, 40, device=DEV).to(BF16)
    block(x).backward(c)
    leaves = [x, block.gate, block.up, block.down]
    values = [t.detach().double() for t in leaves]
    steps = [torch.randn_like(v) for v in values]
    f = lambda e: (plain_block(*[v + e * s for v, s in zip(values, steps)], "gelu") * c.double()).sum()     # noqa: E731
    e = 1e-5
    slope = (f(e) - f(-e)) / (2 * e)
    terms = [(t.grad.double() * s) for t, s in zip(leaves, steps)]
    # Each gradient is off by a few roundings of its own terms; they add up as independent ones do, over tens of thousands of
    # entries: a hundredth of the sum of squares' root is far above that and far below a wrong term.
    size = torch.sqrt(sum((t * t).sum() for t in terms))
    assert abs(sum(t.sum() for t in terms) - slope) <= 0.03 * size


def test_a_captured_training_step_replays_as_the_eager_one():
    torch.manual_seed(6)
    gated = ff.GatedLinear(128, 200)
    down = ff.AdaptersLinear((torch.randn(72, 200, device=DEV) / 14).to(BF16), 3, 8)
    with torch.no_grad():
        down.B.normal_()
    leaves = [gated.gate, gated.up, down.A, down.B]
    x, dy = torch.randn(40, 128, device=DEV).to(BF16), torch.randn(40, 72, device=DEV).to(BF16)
    index = torch.randint(-1, 3, (40,), device=DEV, dtype=torch.int32)

    def step():
        y = down(gated(x), index)
        return (y.detach(), *torch.autograd.grad(y, leaves, dy))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        kept = step()
    for i in range(3):
        x.normal_()
        dy.normal_()
        index.random_(-1, 3)
        want = [t.clone() for t in step()]
        for t in kept:
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(kept, want):
            assert torch.equal(a, c), i
    del graph


def test_two_streams_and_frozen_weights():
    torch.manual_seed(7)
    block = ff.GatedFeedForward(96, 160)
    block.down.requires_grad_(False)
    x = torch.randn(30, 96, device=DEV).to(BF16).requires_grad_()
    dy = torch.randn(30, 96, device=DEV).to(BF16)
    want = torch.autograd.grad(block(x), (x, block.gate, block.up), dy)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(torch.autograd.grad(block(x), (x, block.gate, block.up), dy))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, c) for a, c in zip(g, want))
    # The gradient of a sum is an expanded one.
    g, = torch.autograd.grad(block(x).sum(), x)
    assert torch.equal(g, torch.autograd.grad(block(x), x, torch.ones_like(dy))[0])


def test_the_example_trains_and_decodes():
    gated, down, losses = ff.train(steps=3)
    assert len(losses) == 3 and all(v == v for v in losses) and down.A.grad is not None and down.B.grad is not None
    with torch.no_grad():
        x = torch.randn(2, 256, device=DEV).to(BF16)
        assert down(gated(x), torch.tensor([0, -1], device=DEV, dtype=torch.int32)).shape == (2, 256)


@pytest.mark.parametrize("down,error", [(lambda w: w.float(), TypeError), (lambda w: w.cpu(), ValueError)], ids=["fp32", "on the CPU"])
def test_a_down_projection_that_does_not_fit_is_refused(down, error):
    block = ff.GatedFeedForward(64, 96, 40)
    block.down = torch.nn.Parameter(down(block.down.detach()))
    x = torch.randn(3, 64, device=DEV).to(BF16)
    for mode in (torch.no_grad, torch.enable_grad):
        with mode(), pytest.raises(error):
            block(x)


def test_a_batch_without_tokens():
    """Outputs without rows, and gradients of 0 for what learns."""
    gated, block = ff.GatedLinear(64, 96), ff.GatedFeedForward(64, 96, 40)
    down = ff.AdaptersLinear(torch.randn(40, 96, device=DEV).to(BF16), 2, 4)
    index = torch.empty(0, dtype=torch.int32, device=DEV)
    for module, call in ((gated, gated), (block, block), (down, lambda x: down(gated(x), index))):
        x = torch.empty(0, 64, dtype=BF16, device=DEV, requires_grad=True)
        with torch.no_grad():
            assert call(x).shape[0] == 0
        y = call(x)
        y.sum().backward()
        assert x.grad.shape == (0, 64)
        for p in module.parameters():
            assert p.grad.shape == p.shape and torch.all(p.grad == 0)


def whole(*shape):
    """Whole numbers of -1 to 1: sums of their products are exact in any order, so that plans do not matter to the bits."""
    return torch.randint(-1, 2, shape, device=DEV).to(BF16)


@pytest.mark.parametrize("pad,offset", [(0, 0), (1, 0), (3, 1), (8, 8)])
@pytest.mark.parametrize("tokens", [1, 2, 70])
def test_inputs_and_gradients_that_are_slices(tokens, pad, offset):
    """Rows at any stride and address give the bits of their copies, forward and backward."""
    torch.manual_seed(tokens)
    n_in, n_hidden, n_out = 48, 72, 40
    gated, block = ff.GatedLinear(n_in, n_hidden, "relu"), ff.GatedFeedForward(n_in, n_hidden, n_out, "relu")
    down = ff.AdaptersLinear(whole(n_out, n_hidden + pad + offset)[:, offset:n_hidden + offset], 3, 5)
    with torch.no_grad():
        for p in (*gated.parameters(), *block.parameters(), *down.parameters()):
            p.copy_(whole(*p.shape))
    index = torch.randint(-1, 3, (tokens,), device=DEV, dtype=torch.int32)
    wide_x, wide_dy = whole(tokens, offset + n_in + pad), whole(tokens, offset + n_out + pad)
    for call, leaves in ((lambda x: down(gated(x), index), (*gated.parameters(), *down.parameters())), (block, tuple(block.parameters()))):
        results = []
        for slices in (True, False):
            x, dy = wide_x[:, offset:offset + n_in], wide_dy[:, offset:offset + n_out]
            x, dy = (x, dy) if slices else (x.contiguous().clone(), dy.contiguous().clone())
            x = x.detach().requires_grad_()
            y = call(x)
            results.append((y, *torch.autograd.grad(y, (x, *leaves), dy)))
        assert all(torch.equal(a, c) for a, c in zip(*results))


@pytest.mark.parametrize("n,rank", [(0, 4), (2, 0), (1, 1), (3, 1024)])
def test_projections_without_adapters_and_of_the_largest_rank(n, rank):
    torch.manual_seed(rank)
    down = ff.AdaptersLinear(whole(24, 40), n, rank)
    with torch.no_grad():
        down.A.copy_(whole(n, rank, 40))
        down.B.copy_(whole(n, 24, rank))
    x = whole(9, 40).requires_grad_()
    dy = whole(9, 24)
    index = torch.randint(-1, n, (9,), device=DEV, dtype=torch.int32) if n else torch.zeros(9, dtype=torch.int32, device=DEV)
    y = down(x, index)
    grads = torch.autograd.grad(y, (x, down.A, down.B), dy)
    X, W, A, B = (t.detach().double() for t in (x, down.weight, down.A, down.B))
    want, dx, dA, dB = X @ W.t(), dy.double() @ W, torch.zeros_like(A), torch.zeros_like(B)
    for t, i in enumerate(index.tolist()):
        if n and i >= 0:
            h, dh = X[t] @ A[i].t(), dy[t].double() @ B[i]
            want[t] += h @ B[i].t()
            dx[t] += dh @ A[i]
            dA[i] += torch.outer(dh, X[t])
            dB[i] += torch.outer(dy[t].double(), h)
    for got, v in zip((y.detach(), *grads), (want, dx, dA, dB)):
        assert torch.equal(got, v.to(BF16))


def test_one_leaf_at_a_time():
    """Whatever learns alone gets the gradient that it gets among the others."""
    torch.manual_seed(9)
    gated, block = ff.GatedLinear(48, 72), ff.GatedFeedForward(48, 72)
    down = ff.AdaptersLinear(torch.randn(40, 72, device=DEV).to(BF16), 3, 5)
    with torch.no_grad():
        down.B.normal_()
    index = torch.randint(-1, 3, (33,), device=DEV, dtype=torch.int32)
    x = torch.randn(33, 48, device=DEV).to(BF16)
    for call, modules in ((lambda: down(gated(x), index), (gated, down)), (lambda: block(x), (block,))):
        leaves = [x, *(p for m in modules for p in m.parameters())]
        for t in leaves:
            t.requires_grad_()
        y = call()
        dy = torch.randn_like(y)
        want = torch.autograd.grad(y, leaves, dy, retain_graph=True)
        kept = torch.autograd.grad(y, leaves, dy, create_graph=True)
        assert all(torch.equal(a, c) for a, c in zip(kept, want))
        for i in range(len(leaves)):
            for j, t in enumerate(leaves):
                t.requires_grad_(i == j)
            y2 = call()
            assert torch.equal(y2, y) and torch.equal(torch.autograd.grad(y2, leaves[i], dy)[0], want[i])
        x.requires_grad_(False)
