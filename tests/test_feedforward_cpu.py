"""The feed-forward modules as torch modules, on the CPU: what autograd and the module see of them, with plain products
standing in for the kernels."""
import pytest
import torch

import fused_reference as ref
from paper_2512_13282_amd import binding, feedforward as ff

BF16 = torch.bfloat16


@pytest.fixture
def plain(monkeypatch):
    def gated(x, wg, wu, name="silu", keep=False):
        g, u = x.detach().double() @ wg.detach().double().t(), x.detach().double() @ wu.detach().double().t()
        h = ref.act(name, g)[0] * u
        return (h.to(BF16), g, u) if keep else h.to(BF16)

    def bwd(dh, g, u, name="silu"):
        a, s = ref.act(name, g)
        return dh.double() * u * s, dh.double() * a

    def grad(dy, wd, g, u, name="silu"):
        return (*bwd(dy.double() @ wd.detach().double(), g, u, name), ref.act(name, g)[0] * u)

    d = lambda t: t.detach().double()       # noqa: E731
    stand_ins = {
        "gated_linear": gated, "gated_linear_bwd": bwd, "gated_linear_grad": grad,
        "gated_linear_dx": lambda dg, wg, du, wu: (d(dg) @ d(wg) + d(du) @ d(wu)).to(BF16),
        "gated_linear_dw": lambda dg, du, x, out_dtype: (((d(dg)).t() @ d(x)).to(out_dtype), ((d(du)).t() @ d(x)).to(out_dtype)),
        "linear_dw": lambda dy, x, out_dtype: (d(dy).t() @ d(x)).to(out_dtype),
    }
    for name, fn in stand_ins.items():
        monkeypatch.setattr(binding, name, fn, raising=False)
    monkeypatch.setattr(ff, "_linear", lambda x, W: (d(x) @ d(W).t()).to(BF16))


def test_gradients_and_a_second_derivative(plain):
    torch.manual_seed(0)
    block = ff.GatedFeedForward(24, 40, 16, device="cpu")
    x = torch.randn(6, 24).to(BF16).requires_grad_()
    wanted = (x, block.gate, block.up, block.down)
    once = torch.autograd.grad(block(x).float().pow(2).mean(), wanted)
    kept = torch.autograd.grad(block(x).float().pow(2).mean(), wanted, create_graph=True)
    for a, b in zip(once, kept):
        assert torch.equal(a, b.detach()) and a.dtype == BF16
    with pytest.raises(RuntimeError, match="first derivatives"):
        kept[0].float().pow(2).sum().backward()
    X, wg, wu, wd = (t.detach().double().requires_grad_() for t in wanted)
    y = (torch.nn.functional.silu(X @ wg.t()) * (X @ wu.t())) @ wd.t()
    for got, want in zip(once, torch.autograd.grad(y.pow(2).mean(), (X, wg, wu, wd))):
        assert torch.allclose(got.double(), want, rtol=0.05, atol=0.05 * want.abs().max().item())
    gated = ff.GatedLinear(24, 40, "relu", device="cpu")
    g, = torch.autograd.grad(gated(x).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="first derivatives"):
        g.float().pow(2).sum().backward()


def test_what_learns_and_what_is_saved(tmp_path):
    W = torch.randn(12, 20).to(BF16)
    layer = ff.AdaptersLinear(W, 3, 4)
    assert [n for n, _ in layer.named_parameters()] == ["A", "B"] and not layer.weight.requires_grad
    assert layer.A.shape == (3, 4, 20) and layer.B.shape == (3, 12, 4) and torch.all(layer.B == 0)
    path = tmp_path / "layer.pt"
    torch.save(layer.state_dict(), path)
    other = ff.AdaptersLinear(torch.zeros_like(W), 3, 4, scale=2.0)
    other.load_state_dict(torch.load(path, weights_only=True))
    assert torch.equal(other.weight, W) and torch.equal(other.A, layer.A) and torch.all(other.scale == 1)
    block = ff.GatedFeedForward(20, 12, device="cpu")
    assert sorted(block.state_dict()) == ["down", "gate", "up"] and block.down.shape == (20, 12)
    assert {t.device.type for t in block.to("meta").state_dict().values()} == {"meta"}


def test_modules_are_reached_beside_their_operators():
    from paper_2512_13282_amd import adapters, ffn
    assert ffn.GatedFeedForward is ff.GatedFeedForward and ffn.GatedLinear is ff.GatedLinear and adapters.AdaptersLinear is ff.AdaptersLinear
    for module in (ffn, adapters):
        with pytest.raises(AttributeError):
            module.NoSuchModule


class _OnGpu:
    """Stands for a matrix on a GPU: its address must not be taken."""
    is_cuda = True

    def __init__(self, *shape, dtype=BF16, index=0):
        self.shape, self.dtype, self.index, self.device = torch.Size(shape), dtype, index, torch.device("cuda", index)

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.index

    def data_ptr(self):
        pytest.fail("the address of an operand that has to be refused was taken")


@pytest.mark.parametrize("x,W,error", [
    (torch.zeros(3, 8, dtype=BF16), torch.zeros(5, 8), TypeError),                       # an fp32 weight
    (torch.zeros(3, 8), torch.zeros(5, 8, dtype=BF16), TypeError),
    (_OnGpu(3, 8), torch.zeros(5, 8), TypeError),
    (_OnGpu(3, 8), torch.zeros(5, 8, dtype=BF16), ValueError),                           # a weight that is not on the GPU
    (_OnGpu(3, 8), _OnGpu(5, 8, index=1), ValueError),                                   # ... on another one
    (torch.zeros(3, 8, dtype=BF16), torch.zeros(5, 8, dtype=BF16), ValueError),
    (_OnGpu(3, 8), _OnGpu(5, 9), ValueError),
    (_OnGpu(3, 8), _OnGpu(5, 8, 1), ValueError),
    (_OnGpu(2, 3, 8), _OnGpu(5, 8), ValueError),
], ids=lambda v: v.__name__ if isinstance(v, type) else f"{type(v).__name__}-{'x'.join(map(str, v.shape))}-{v.dtype}")
def test_the_down_projection_refuses_what_is_not_a_bf16_matrix_on_its_gpu(x, W, error, monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda *_, **__: pytest.fail("a result was allocated for operands that have to be refused"))
    with pytest.raises(error):
        ff._linear(x, W)


@pytest.mark.parametrize("mode", [torch.no_grad, torch.enable_grad])
def test_a_tangent_is_refused_and_not_dropped(plain, mode, monkeypatch):
    """Forward-mode derivatives, of an input or of a parameter, with and without a graph for the backward pass."""
    from torch.autograd import forward_ad
    monkeypatch.setattr(binding, "linear_adapters", lambda x, W, held, index, keep=False:
                        (x.detach() @ W.t(), x.detach() @ held.A[0].t()) if keep else x.detach() @ W.t(), raising=False)
    x, index = torch.randn(6, 24).to(BF16), torch.zeros(6, dtype=torch.int32)
    adapters = ff.AdaptersLinear(torch.randn(16, 24).to(BF16), 2, 4)
    calls = [(ff.GatedLinear(24, 40, device="cpu"), ()), (ff.GatedFeedForward(24, 40, device="cpu"), ()), (adapters, (index,))]
    for module, rest in calls:
        with mode(), forward_ad.dual_level():
            assert module(x, *rest).shape[0] == 6
            with pytest.raises(RuntimeError, match="forward"):
                module(forward_ad.make_dual(x, torch.ones_like(x)), *rest)
            for name, p in [*module.named_parameters(), *module.named_buffers()]:
                dual = forward_ad.make_dual(p.detach(), torch.ones_like(p))
                with pytest.raises(RuntimeError, match="forward"):
                    torch.func.functional_call(module, {name: dual}, (x, *rest))


@pytest.mark.parametrize("default", [torch.float32, torch.float64, BF16])
def test_scales_are_fp32_whatever_they_are_made_of_and_the_module_becomes(default):
    torch.set_default_dtype(default)
    try:
        W = torch.randn(12, 20).to(BF16)
        whole, third = ff.AdaptersLinear(W, 3, 4, scale=2), ff.AdaptersLinear(W, 3, 4, scale=0.3)
    finally:
        torch.set_default_dtype(torch.float32)
    want = torch.full((3,), 0.3, dtype=torch.float32)
    assert whole.scale.dtype == torch.float32 and torch.all(whole.scale == 2) and torch.equal(third.scale, want)
    # The usual conversions of a model, alone and inside another module, keep the value and not only the type.
    for convert in (lambda m: m.to(BF16), lambda m: m.bfloat16(), lambda m: m.half().to(BF16), lambda m: m.double().to(BF16),
                    lambda m: torch.nn.Sequential(m).to(torch.device("cpu"), BF16)[0]):
        layer = convert(ff.AdaptersLinear(W, 3, 4, scale=0.3))
        assert torch.equal(layer.scale, want) and layer.A.dtype == BF16 and layer.weight.dtype == BF16
        assert "scale" in layer.state_dict() and "scale" in dict(layer.named_buffers())
    layer = third.to("meta", BF16)
    assert layer.scale.device.type == "meta" and layer.scale.dtype == torch.float32
    assert layer.to_empty(device="cpu").scale.shape == (3,)


def test_scales_that_are_to_learn_are_refused(monkeypatch):
    """They have no gradient: left out of the backward pass without a word they would never move."""
    monkeypatch.setattr(binding, "linear_adapters", lambda x, W, held, index, keep=False:
                        (x.detach() @ W.t(), x.detach() @ held.A[0].t()) if keep else x.detach() @ W.t(), raising=False)
    layer = ff.AdaptersLinear(torch.randn(12, 20).to(BF16), 2, 4)
    x, index = torch.randn(6, 20).to(BF16), torch.zeros(6, dtype=torch.int32)
    layer.scale.requires_grad_()
    with pytest.raises(RuntimeError, match="scales"):
        layer(x, index)
    with torch.no_grad():
        assert layer(x, index).shape == (6, 12)
    layer.scale.requires_grad_(False)
    assert layer(x, index).requires_grad


def test_an_empty_matrix_has_no_strides_that_matter():
    """The gradient of a sum over no tokens is an expanded matrix without rows, and contiguous() leaves its strides of 0."""
    from paper_2512_13282_amd import adapters, mx
    x = torch.zeros(1).expand(0, 96).contiguous()
    assert x.stride() == (0, 0)
    assert mx._ld(x.stride(), *x.shape) == 96
    for stride in ((0, 0), (1, 5), (96, 1)):
        assert mx._ld(stride, 0, 96) == 96 and mx._ld(stride, 5, 0) == 1
    with pytest.raises(ValueError):
        mx._ld((0, 0), 1, 96)
    assert adapters._stack(torch.zeros(1).expand(0, 8, 96), 0, 8, 96)[0] == 96
