"""The adapter layer as a torch module, on the CPU: what autograd and the module see of it, with plain
products standing in for the kernels."""
import pytest
import torch

from paper_2512_13282_amd import adapter, binding

N_IN, N_OUT, RANK, TOKENS = 40, 24, 3, 5


def base(seed=0, n_in=N_IN, n_out=N_OUT):
    """A 4-bit weight as packing lays it out: rows of codes 16 bytes or a multiple apart."""
    gen = torch.Generator()
    gen.manual_seed(seed)
    width = (n_in + 1) // 2
    codes = torch.empty_strided((n_out, width), (-(-width // 16) * 16, 1), dtype=torch.uint8)
    codes.copy_(torch.randint(0, 256, codes.shape, generator=gen))
    return binding.MxMatrix(codes, torch.full((n_out, (n_in + 31) // 32), 124 + seed, dtype=torch.uint8), n_in)


GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def values(W):
    q = torch.stack((W.codes & 15, W.codes >> 4), 2).reshape(W.codes.shape[0], -1)[:, :W.cols].long()
    v = torch.where(q >= 8, -GRID[q & 7], GRID[q & 7])
    return v * torch.exp2(W.scales.float() - 127).repeat_interleave(32, 1)[:, :W.cols]


@pytest.fixture
def plain(monkeypatch):
    """The kernels' results by plain products; an "8-bit" matrix keeps its values as they are."""
    pairs = {
        "mm_bf16_f32": lambda a, b: a.detach().float() @ b.detach().float(),
        "linear_mx4": lambda a, W, out_dtype=torch.bfloat16: (a.detach().float() @ values(W).t()).to(out_dtype),
        "linear_mx4_dx": lambda g, W, out_dtype=torch.bfloat16: (g.detach().float() @ values(W)).to(out_dtype),
        "pack_mx8": lambda x: binding.MxMatrix(x.detach().clone(), torch.empty(0), x.shape[1]),
        "linear_mx8_dw": lambda g, X, out_dtype=torch.float32: (g.detach().t().float() @ X.codes.float()).to(out_dtype),
    }
    for name, fn in pairs.items():
        monkeypatch.setattr(binding, name, fn, raising=False)


def layer_and_input():
    torch.manual_seed(1)
    layer = adapter.AdapterLinear(base(), RANK)
    with torch.no_grad():
        layer.B.copy_(torch.randn(N_OUT, RANK))
    return layer, torch.randn(TOKENS, N_IN).to(torch.bfloat16).requires_grad_()


def test_a_second_derivative_raises(plain):
    layer, x = layer_and_input()
    loss = layer(x).float().pow(2).mean()
    g, = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives"):
        (loss + g.float().pow(2).sum()).backward()              # a gradient penalty
    # The gradient of a plain sum, whose own incoming gradient is a constant.
    g, = torch.autograd.grad(layer(x).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives"):
        g.float().pow(2).sum().backward()
    for p in (layer.A, layer.B):
        g, = torch.autograd.grad(layer(x).float().pow(2).mean(), p, create_graph=True)
        with pytest.raises(RuntimeError, match="first derivatives"):
            g.float().pow(2).sum().backward()


def test_first_derivatives_do_not_depend_on_the_graph_kept(plain):
    layer, x = layer_and_input()
    wanted = (x, layer.A, layer.B)
    once = torch.autograd.grad(layer(x).float().pow(2).mean(), wanted)
    kept = torch.autograd.grad(layer(x).float().pow(2).mean(), wanted, create_graph=True)
    for a, b in zip(once, kept):
        assert torch.equal(a, b.detach())
    w = values(layer.weight)
    xf, A, B = (t.detach().float().requires_grad_() for t in wanted)
    y = xf @ w.t() + (xf @ A.t()) @ B.t()
    for got, want in zip(once, torch.autograd.grad(y.pow(2).mean(), (xf, A, B))):
        # bf16 activations and gradients on the way: a few roundings of 2^-9 against the terms.
        assert torch.allclose(got.float(), want, rtol=0.05, atol=0.05 * want.abs().max().item())


def test_a_gradient_that_is_a_constant_stays_one(plain):
    """With the adapter frozen and a constant gradient coming in, dx depends on nothing that learns."""
    layer, x = layer_and_input()
    layer.A.requires_grad_(False)
    layer.B.requires_grad_(False)
    g, = torch.autograd.grad(layer(x).sum(), x, create_graph=True)
    assert not g.requires_grad


def same(a, b):
    return torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales) and a.cols == b.cols


def test_a_saved_layer_holds_its_weight(plain, tmp_path):
    layer, x = layer_and_input()
    path = tmp_path / "layer.pt"
    torch.save(layer.state_dict(), path)
    other = adapter.AdapterLinear(base(seed=3), RANK)
    assert not same(other.weight, layer.weight)
    other.load_state_dict(torch.load(path, weights_only=True))
    assert same(other.weight, layer.weight)
    with torch.no_grad():
        assert torch.equal(other(x), layer(x))
    # An adapter alone, or one over a weight of another shape, is not taken for a layer.
    with pytest.raises(RuntimeError):
        other.load_state_dict({"A": layer.A, "B": layer.B})
    with pytest.raises(RuntimeError):
        adapter.AdapterLinear(base(n_in=38), RANK).load_state_dict(layer.state_dict())


@pytest.mark.parametrize("move", [lambda m: m.to("meta"), lambda m: m.to_empty(device="meta"),
                                  lambda m: torch.nn.Sequential(m).to("meta")[0]])
def test_the_weight_moves_with_the_layer(move):
    layer = move(adapter.AdapterLinear(base(), RANK))
    assert {t.device.type for t in (*layer.weight[:2], layer.A, layer.B)} == {"meta"}
    # Rows stay where the products read them as they lie.
    assert layer.weight.codes.stride() == (32, 1) and layer.weight.cols == N_IN


def test_rows_that_follow_each_other_are_laid_out_once():
    Q = base()
    layer = adapter.AdapterLinear(binding.MxMatrix(Q.codes.contiguous(), Q.scales, Q.cols), RANK)
    assert layer.weight.codes.stride() == (32, 1) and same(layer.weight, Q)
    layer.weight = binding.MxMatrix(base(seed=2).codes.contiguous(), base(seed=2).scales, N_IN)
    assert layer.weight.codes.stride() == (32, 1) and same(layer.weight, base(seed=2))
    layer.weight = Q
    layer.load_state_dict({k: v.clone().contiguous() for k, v in layer.state_dict().items()}, assign=True)
    assert same(layer.weight, Q)
    assert same(adapter.AdapterLinear(base(n_in=1), 1).weight, base(n_in=1))


def test_only_the_adapter_learns():
    layer = adapter.AdapterLinear(base(), RANK)
    assert [n for n, _ in layer.named_parameters()] == ["A", "B"]
    assert not layer.weight.codes.requires_grad


@pytest.mark.parametrize("mode", [torch.no_grad, torch.enable_grad])
def test_a_tangent_is_refused_and_not_dropped(plain, mode):
    """Forward-mode derivatives, with and without a graph for the backward pass."""
    from torch.autograd import forward_ad
    layer, x = layer_and_input()
    x = x.detach()
    with mode(), forward_ad.dual_level():
        assert layer(x).shape == (TOKENS, N_OUT)
        with pytest.raises(RuntimeError, match="forward"):
            layer(forward_ad.make_dual(x, torch.ones_like(x)))
        for name, p in layer.named_parameters():
            with pytest.raises(RuntimeError, match="forward"):
                torch.func.functional_call(layer, {name: forward_ad.make_dual(p.detach(), torch.ones_like(p))}, (x,))
