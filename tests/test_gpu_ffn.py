"""The gated feed-forward kernels against their definitions in 64 bits, within the bounds of their fp32 sums and their
one rounding (fused_reference.py)."""
import zlib

import pytest
import torch

import fused_reference as ref
from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import ffn

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF16 = torch.bfloat16


def matrix(gen, rows, cols, scale=1.0, pad=0, offset=0):
    """A bf16 matrix in a larger buffer of NaN: rows `pad` elements apart from contiguous, `offset` elements in."""
    x = (torch.randn(rows, cols, generator=gen) * scale).to(BF16)
    buf = torch.full((offset + rows * (cols + pad) + 8,), float("nan"), dtype=BF16)
    view = buf[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] if rows and cols else buf[:0].view(rows, cols)
    view.copy_(x)
    dev = buf.to(DEV)
    return dev[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] if rows and cols else dev[:0].view(rows, cols)


def generator(*key):
    gen = torch.Generator()
    gen.manual_seed(zlib.crc32(repr(key).encode()))
    return gen


# M, N, K, pad, offset of the operands (elements)
SIZES = [(1, 8, 8, 0, 0), (1, 1, 1, 0, 0), (3, 7, 5, 0, 0), (17, 33, 65, 0, 0), (64, 128, 64, 0, 0), (65, 129, 72, 8, 8), (37, 131, 129, 1, 3),
         (100, 264, 320, 0, 0), (130, 250, 1000, 8, 0), (257, 520, 136, 0, 0), (300, 513, 511, 5, 1), (1, 1000, 2048, 0, 0),
         (16, 512, 4104, 0, 0), (511, 264, 64, 0, 0),
         # More tiles than compute units: whole ones, and slices of the rest.
         (1100, 2200, 328, 0, 0), (4340, 4100, 264, 0, 4), (2100, 8200, 72, 0, 0), (72, 4100, 4340, 0, 0)]
ids = dict(ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))


def configurations(op):
    found = []
    for c in range(64):
        if ffn.ffn_force_plan(op, c) == b.GEMM_OK:
            found.append(c)
    ffn.ffn_force_plan(op)
    return found


def plans(op, M, N, K, splits=(1, 3)):
    """Every configuration that takes the sizes, forced with each number of slices; the library's own choice first."""
    yield None
    try:
        for config in configurations(op):
            for split in splits:
                assert ffn.ffn_force_plan(op, config, split) == b.GEMM_OK
                try:
                    plan = ffn.ffn_plan(op, M, N, K)
                except b.GemmError as e:
                    assert e.status == b.GEMM_ERR_UNSUPPORTED
                    continue
                if split == 1 or plan["split_k"] > 1:
                    yield plan
    finally:
        ffn.ffn_force_plan(op)


@pytest.mark.parametrize("size", SIZES, **ids)
def test_gated(size):
    M, N, K, pad, offset = size
    gen = generator("gated", *size)
    x, wg, wu = matrix(gen, M, K, 1.0, pad, offset), matrix(gen, N, K, K ** -0.5, pad, offset), matrix(gen, N, K, K ** -0.5, pad, offset)
    name = ref.ACTIVATIONS[(M + N) % 4]
    want = ref.gated(x, wg, wu, name)
    for plan in plans(ffn.FFN_OP_GATED, M, N, K):
        print(size, plan, flush=True)
        got = b.gated_linear(x, wg, wu, name, keep=True)
        for g, w, what in zip(got, want, "HGU"):
            ref.assert_within(g, w, f"{what} {plan}")
        assert torch.equal(b.gated_linear(x, wg, wu, name), got[0])


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_activations_over_their_range(name):
    """Sums that are exact: G takes values from 2^-14 to 2^126 of both signs, U is 1."""
    e = torch.arange(-14, 126, dtype=torch.float64)
    g = torch.cat((2.0 ** e, 1.5 * 2.0 ** e, torch.linspace(-12, 12, 97).to(BF16).double()))
    g = torch.cat((g, -g)).to(BF16)
    N = g.numel()
    x = torch.zeros(2, 8, dtype=BF16)
    x[:, 0] = 1
    wg, wu = torch.zeros(N, 8, dtype=BF16), torch.zeros(N, 8, dtype=BF16)
    wg[:, 0], wu[:, 0] = g, 1
    x, wg, wu = x.to(DEV), wg.to(DEV), wu.to(DEV)
    H, G, U = b.gated_linear(x, wg, wu, name, keep=True)
    assert torch.equal(G[1].cpu(), g)
    a, s = ref.act(name, G.double())
    fine = a.abs() >= 2.0 ** -100           # below: flushed, and the definition's own value is no bf16 number
    assert torch.all(((H.double() - a).abs() <= 2.0 ** -8 * a.abs() + ref.ACT_ERROR * (1 + a.abs()))[fine])
    assert torch.all(H[~fine].double().abs() <= 2.0 ** -99)
    wd = torch.zeros(8, N, dtype=BF16, device=DEV)
    wd[0] = 1
    dG, dU, H2 = b.gated_linear_grad(x, wd, G, U, name)
    assert torch.equal(H2, H) and torch.equal(dU, H)
    assert torch.all((dG.double() - s).abs() <= 2.0 ** -8 * s.abs() + ref.SLOPE_ERROR * (1 + s.abs()))


@pytest.mark.parametrize("size", SIZES, **ids)
def test_grad(size):
    M, N, K, pad, offset = size
    gen = generator("grad", *size)
    dy, wd = matrix(gen, M, K, 1.0, pad, offset), matrix(gen, K, N, K ** -0.5, pad, offset)
    g, u = matrix(gen, M, N, 2.0, pad, offset), matrix(gen, M, N, 1.0, pad, offset)
    name = ref.ACTIVATIONS[(M + K) % 4]
    want = ref.grad(dy, wd, g, u, name)
    for plan in plans(ffn.FFN_OP_GRAD, M, N, K):
        print(size, plan, flush=True)
        for got, w, what in zip(b.gated_linear_grad(dy, wd, g, u, name), want, ("dG", "dU", "H")):
            ref.assert_within(got, w, f"{what} {plan}")


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, **ids)
def test_dx(size, dtype):
    M, N, K, pad, offset = size
    gen = generator("dx", *size)
    dg, du = matrix(gen, M, K, 1.0, pad, offset), matrix(gen, M, K, 1.0, pad, 0)
    wg, wu = matrix(gen, K, N, K ** -0.5, pad, 0), matrix(gen, K, N, K ** -0.5, pad, offset)
    want = ref.dx(dg, wg, du, wu, dtype)
    for plan in plans(ffn.FFN_OP_DX, M, N, K):
        print(size, plan, flush=True)
        ref.assert_within(b.gated_linear_dx(dg, wg, du, wu, out_dtype=dtype), want, f"dX {plan}")


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, **ids)
def test_dw(size, dtype):
    K, N, M, pad, offset = size              # tokens, inputs, outputs
    gen = generator("dw", *size)
    dg, du, x = matrix(gen, K, M, 1.0, pad, offset), matrix(gen, K, M, 1.0, pad, 0), matrix(gen, K, N, 1.0, pad, offset)
    want = ref.dw(dg, x, dtype), ref.dw(du, x, dtype)
    for plan in plans(ffn.FFN_OP_GATED_DW, M, N, K):
        print(size, plan, flush=True)
        for got, w, what in zip(b.gated_linear_dw(dg, du, x, out_dtype=dtype), want, ("dWg", "dWu")):
            ref.assert_within(got, w, f"{what} {plan}")
    for plan in plans(ffn.FFN_OP_DW, M, N, K):
        ref.assert_within(b.linear_dw(dg, x, out_dtype=dtype), want[0], f"dW {plan}")


def test_results_leave_their_padding():
    gen = generator("padding")
    x, wg, wu = matrix(gen, 70, 96), matrix(gen, 133, 96), matrix(gen, 133, 96)
    buf = torch.full((70, 140), 7.0, dtype=BF16, device=DEV)
    H = b.gated_linear(x, wg, wu, out=buf[:, :133])
    assert torch.equal(H, b.gated_linear(x, wg, wu)) and torch.all(buf[:, 133:] == 7)
    for dtype in (torch.float32, BF16):
        buf = torch.full((133, 100), 7.0, dtype=dtype, device=DEV)
        b.linear_dw(H, x, out=buf[:, :96])
        assert torch.equal(buf[:, :96], b.linear_dw(H, x, out_dtype=dtype)) and torch.all(buf[:, 96:] == 7)
        buf = torch.full((70, 100), 7.0, dtype=dtype, device=DEV)
        b.gated_linear_dx(H, wg, H, wu, out=buf[:, :96])
        assert torch.equal(buf[:, :96], b.gated_linear_dx(H, wg, H, wu, out_dtype=dtype)) and torch.all(buf[:, 96:] == 7)


def test_empty_sums_and_results():
    e = lambda r, c: torch.empty(r, c, dtype=BF16, device=DEV)      # noqa: E731
    for got in (*b.gated_linear(e(5, 0), e(6, 0), e(6, 0), keep=True), *b.gated_linear_dw(e(0, 5), e(0, 5), e(0, 6)),
                b.linear_dw(e(0, 5), e(0, 6)), b.gated_linear_dx(e(5, 0), e(0, 6), e(5, 0), e(0, 6))):
        assert got.shape == (5, 6) and torch.all(got == 0)
    g, u = torch.randn(5, 6, device=DEV).to(BF16), torch.randn(5, 6, device=DEV).to(BF16)
    dg, du, h = b.gated_linear_grad(e(5, 0), e(0, 6), g, u)
    assert torch.all(dg == 0) and torch.all(du == 0)
    ref.assert_within(h, ref.grad(e(5, 0), e(0, 6), g, u, "silu")[2])
    assert b.gated_linear(e(0, 8), e(6, 8), e(6, 8)).shape == (0, 6) and b.gated_linear(e(5, 8), e(0, 8), e(0, 8)).shape == (5, 0)
    assert b.linear_dw(e(7, 0), e(7, 6)).shape == (0, 6)


def test_what_is_not_finite_stays_in_its_row_and_column():
    gen = generator("nan")
    x, wg, wu = matrix(gen, 80, 200), matrix(gen, 150, 200), matrix(gen, 150, 200)
    clean = b.gated_linear(x, wg, wu)
    x2, wg2 = x.clone(), wg.clone()
    x2[3, 7] = float("nan")
    x2[70, 199] = float("inf")
    wg2[140, 0] = float("nan")
    H = b.gated_linear(x2, wg2, wu)
    rows = torch.ones(80, dtype=torch.bool, device=DEV)
    rows[3] = rows[70] = False
    cols = torch.ones(150, dtype=torch.bool, device=DEV)
    cols[140] = False
    assert torch.equal(H[rows][:, cols], clean[rows][:, cols])
    assert torch.all(torch.isnan(H[3])) and torch.all(torch.isnan(H[:, 140])) and not torch.any(torch.isfinite(H[70]) & (H[70] != 0))


@pytest.mark.parametrize("op", range(5))
def test_slices_give_the_same_bits_captured_and_on_every_stream(op):
    """A captured call on a stream without counters, replayed among eager calls, and calls on several streams at once."""
    gen = generator("bits", op)
    M, N, K = 70, 150, 1000
    mk = {0: lambda: b.gated_linear(x, w1, w2, keep=True), 1: lambda: b.gated_linear_grad(x, v1, g, u),
          2: lambda: b.gated_linear_dx(x, v1, y, v2, out_dtype=torch.float32),
          3: lambda: b.gated_linear_dw(t1, t2, t3), 4: lambda: b.linear_dw(t1, t3, out_dtype=BF16)}[op]
    x, y = matrix(gen, M, K), matrix(gen, M, K)
    w1, w2, v1, v2 = matrix(gen, N, K), matrix(gen, N, K), matrix(gen, K, N, pad=2), matrix(gen, K, N)
    g, u = matrix(gen, M, N), matrix(gen, M, N)
    t1, t2, t3 = matrix(gen, K, M, pad=2), matrix(gen, K, M, pad=2), matrix(gen, K, N, pad=2)
    call = lambda: (lambda r: r if isinstance(r, tuple) else (r,))(mk())     # noqa: E731
    for plan in plans(op, *((M, N, K)), splits=(1, 4)):
        torch.cuda.synchronize()
        assert b.gemm_release_workspace() == b.GEMM_OK
        s = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            held = call()
        for i in range(3):
            for t in (x, y, t1, t2):
                t.normal_()
            want = call()
            for h in held:
                h.fill_(7.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, c in zip(held, want):
                assert torch.equal(a, c), (plan, i)
        results = []
        streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
        for _ in range(2):
            for q in streams:
                with torch.cuda.stream(q):
                    results.append(call())
        torch.cuda.synchronize()
        for r in results:
            for a, c in zip(r, want):
                assert torch.equal(a, c), plan
        del graph
    torch.cuda.synchronize()
    assert b.gemm_release_workspace() == b.GEMM_OK


@pytest.mark.parametrize("size", [(1, 8, 0), (3, 7, 1), (70, 133, 5), (300, 1000, 8)], **ids)
@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_gradients_from_that_of_h(size, name):
    M, N, pad = size
    gen = generator("bwd", *size)
    dh, g, u = matrix(gen, M, N, 1.0, pad, 0), matrix(gen, M, N, 2.0, pad, pad % 2), matrix(gen, M, N, 1.0, pad, 0)
    d = dh.double()
    a, s = ref.act(name, g.double())
    dG, dU = b.gated_linear_bwd(dh, g, u, name)
    for got, v, e in ((dG, d * u.double() * s, (d * u.double()).abs() * ref.SLOPE_ERROR * (1 + s.abs())),
                      (dU, d * a, d.abs() * ref.ACT_ERROR * (1 + a.abs()))):
        ref.assert_within(got, (v, ref.rounded(v, e + 2.0 ** -22 * v.abs(), BF16)))


def test_gradients_without_h():
    gen = generator("no h")
    dy, wd, g, u = matrix(gen, 70, 96), matrix(gen, 96, 133), matrix(gen, 70, 133), matrix(gen, 70, 133)
    want = b.gated_linear_grad(dy, wd, g, u)
    dG, dU = torch.empty_like(want[0]), torch.empty_like(want[1])
    rc = ffn.ffn_gated_grad_bf16(70, 133, 96, dy.data_ptr(), 96, wd.data_ptr(), 133, g.data_ptr(), 133, u.data_ptr(), 133, 0, dG.data_ptr(), 133,
                                 dU.data_ptr(), 133, 0, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == b.GEMM_OK and torch.equal(dG, want[0]) and torch.equal(dU, want[1])


def test_a_workspace_that_cannot_be_had(monkeypatch):
    """Nothing is queued, and a later call allocates afresh."""
    gen = generator("memory")
    x, w = matrix(gen, 30, 1000), matrix(gen, 200, 1000)
    try:
        assert ffn.ffn_force_plan(ffn.FFN_OP_GATED, 0, 4) == b.GEMM_OK
        want = b.gated_linear(x, w, w)
        torch.cuda.synchronize()
        assert b.gemm_release_workspace() == b.GEMM_OK
        out = torch.full_like(want, 7.0)
        monkeypatch.setenv("GEMM_MI355X_TEST_FAIL_WORKSPACE", "1")
        with pytest.raises(b.GemmError) as e:
            b.gated_linear(x, w, w, out=out)
        assert e.value.status == b.GEMM_ERR_NO_MEMORY
        torch.cuda.synchronize()
        assert torch.all(out == 7)
        monkeypatch.delenv("GEMM_MI355X_TEST_FAIL_WORKSPACE")
        assert torch.equal(b.gated_linear(x, w, w, out=out), want)
    finally:
        ffn.ffn_force_plan(ffn.FFN_OP_GATED)


def test_rows_far_apart():
    """Strides past 4 MiB are copied first, and offsets past 2 GiB reached."""
    gen = generator("far")
    small, wg = matrix(gen, 260, 64), matrix(gen, 40, 64)
    buf = torch.empty(260 * (1 << 22) + 64, dtype=BF16, device=DEV)
    x = buf.as_strided((260, 64), (1 << 22, 1))
    x.copy_(small)
    assert torch.equal(b.gated_linear(x, wg, wg), b.gated_linear(small, wg, wg))
    assert torch.equal(b.linear_dw(x, x), b.linear_dw(small, small))
    near = buf.as_strided((260, 64), (1 << 21, 1))                # 4 MiB apart: as they lie
    near.copy_(small)
    assert torch.equal(b.gated_linear(near, wg, wg), b.gated_linear(small, wg, wg))


def test_results_past_four_gib():
    """Offsets of results and operands past 32 bits: the last rows are those of a call on them alone."""
    gen = generator("large")
    M, N, K = 70000, 33000, 40
    wg = matrix(gen, N, K)
    x = torch.randn(M, K, device=DEV).to(BF16)
    H = b.gated_linear(x, wg, wg)
    assert torch.equal(H[-300:], b.gated_linear(x[-300:].clone(), wg, wg)) and torch.equal(H[:300], b.gated_linear(x[:300].clone(), wg, wg))
    # H as an operand along the sum and across it.
    dX = b.gated_linear_dx(H, wg, H, wg, out_dtype=torch.float32)
    ref.assert_within(dX[-40:], ref.dx(H[-40:], wg, H[-40:], wg, torch.float32))
    dW = b.linear_dw(H, x)
    ref.assert_within(dW[-8:], ref.dw(H[:, -8:], x, torch.float32))
    dG, dU = b.gated_linear_bwd(H, H, H)
    small = b.gated_linear_bwd(H[-5:].clone(), H[-5:].clone(), H[-5:].clone())
    assert torch.equal(dG[-5:], small[0]) and torch.equal(dU[-5:], small[1])


def tail_bounds(name, g):
    """act(g) and act'(g) in 64 bits, each with a bound that is relative to the terms it is the sum of.

    With t = |z| for p = 1 / (1 + e^-z) (silu, gelu_tanh): z is off by four roundings, 2^-24 |z| each, and so the exponent; 2^x, 1 / x
    and the products add single steps of 2^-23.  With t = g^2 for gelu: erfc of an argument that is off by 1.5 2^-24 of itself moves by g^2 + 1
    times that, and erfc itself is taken to be good to 16 steps, 2^-19.  (1 + t) 2^-19 covers each.  A bf16 result adds 2^-8."""
    if name == "relu":
        a, s = ref.act(name, g)
        return (a, 2.0 ** -8 * a), (s, 2.0 ** -8 * s)
    if name == "gelu":
        p, slope, t = 0.5 * torch.special.erfc(-g / 2 ** 0.5), torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5, g * g
    else:
        c = 2 * (2 / torch.pi) ** 0.5
        z, dz = (g, 1.0) if name == "silu" else (c * (g + 0.044715 * g ** 3), c * (1 + 3 * 0.044715 * g * g))
        p, slope, t = torch.sigmoid(z), torch.sigmoid(z) * torch.sigmoid(-z) * dz, z.abs()
    a, s = g * p, p + g * slope
    off = 2.0 ** -19 * (1 + t)
    return (a, (2.0 ** -8 + off) * a.abs()), (s, 2.0 ** -8 * s.abs() + off * (p + g.abs() * slope))


@pytest.mark.parametrize("name", ref.ACTIVATIONS)
def test_activations_in_their_tails(name):
    """Small values of act and act' keep their bits down to 2^-100; below that they may be 0."""
    g = torch.unique(torch.cat((torch.linspace(-80, 80, 3201), torch.linspace(-14, 14, 2801), torch.linspace(-1.5, 1.5, 301))).to(BF16))
    N = g.numel()
    x, wg, wu = torch.zeros(2, 8, dtype=BF16), torch.zeros(N, 8, dtype=BF16), torch.zeros(N, 8, dtype=BF16)
    x[:, 0], wg[:, 0], wu[:, 0] = 1, g, 1
    x, wg, wu, wd = x.to(DEV), wg.to(DEV), wu.to(DEV), torch.zeros(8, N, dtype=BF16, device=DEV)
    wd[0] = 1
    (a, ea), (s, es) = tail_bounds(name, g.to(DEV).double())

    def within(got, want, bound, what):
        off, small = (got.double() - want).abs(), want.abs() < 2.0 ** -100
        assert torch.all((off <= bound)[~small.expand_as(off)]), (what, (off / (bound + 1e-300))[~small.expand_as(off)].max().item())
        assert torch.all(got.double().abs()[small.expand_as(off)] <= 2.0 ** -99), what

    for plan in plans(ffn.FFN_OP_GATED, 2, N, 8, splits=(1,)):
        H, G, U = b.gated_linear(x, wg, wu, name, keep=True)
        within(H, a, ea, ("act", plan))
    one = torch.ones_like(G)
    for what, got in (("grad", b.gated_linear_grad(x, wd, G, U, name)), ("bwd", (*b.gated_linear_bwd(one, G, U, name), H))):
        within(got[0], s, es, ("slope", what))
        within(got[1], a, ea, ("act of the gradient", what))
        within(got[2], a, ea, ("H again", what))


# M, N, K of the result: whole rounds of 256 x 256 tiles leave more behind by columns than by rows, so the lower tiles take the rows
# after them (of the second gradient, where there are two).
ROW_TAILS = [(23040, 700, 72), (22950, 651, 40)]


def leaves_rows(M, cols, pairs):
    """Whether tiles of 256 rows and `cols` columns, walked in whole rounds of 256, end with lower tiles over rows."""
    tm, tn = -(-M // 256) * pairs, -(-cols // 256)
    full = tm * tn // 256 * 256
    return 0 < full < tm * tn and full // tm * tm < full // tn * tn


@pytest.mark.parametrize("config", [4, 5])
@pytest.mark.parametrize("size", ROW_TAILS, **ids)
def test_lower_tiles_over_the_last_rows(size, config):
    M, N, K = size
    gen = generator("row tails", *size)
    x, w, v = matrix(gen, M, K), matrix(gen, N, K, K ** -0.5), matrix(gen, K, N, K ** -0.5)
    half, u = N // 2, matrix(gen, M, N)
    t, y = matrix(gen, K, M), matrix(gen, K, N)
    first, second = matrix(gen, K, M // 2), matrix(gen, K, M // 2)
    assert leaves_rows(M, N, 1) and leaves_rows(M // 2, N, 2) and leaves_rows(M, 2 * half, 1)
    calls = {
        ffn.FFN_OP_GATED: (lambda: b.gated_linear(x, w[:half], w[half:2 * half], "gelu", keep=True), lambda: ref.gated(x, w[:half], w[half:2 * half], "gelu")),
        ffn.FFN_OP_GRAD: (lambda: b.gated_linear_grad(x, v, u, u, "silu"), lambda: ref.grad(x, v, u, u, "silu")),
        ffn.FFN_OP_DX: (lambda: (b.gated_linear_dx(x, v, x, v),), lambda: (ref.dx(x, v, x, v, BF16),)),
        ffn.FFN_OP_GATED_DW: (lambda: b.gated_linear_dw(first, second, y), lambda: (ref.dw(first, y, torch.float32), ref.dw(second, y, torch.float32))),
        ffn.FFN_OP_DW: (lambda: (b.linear_dw(t, y),), lambda: (ref.dw(t, y, torch.float32),)),
    }
    for op, (call, want) in calls.items():
        try:
            assert ffn.ffn_force_plan(op, config, 1) == b.GEMM_OK
            print(size, config, op, flush=True)
            got = call()
        finally:
            ffn.ffn_force_plan(op)
        for g, w64 in zip(got, want()):
            ref.assert_within(g, w64, f"op {op}")


@pytest.mark.parametrize("size", [(11008, 4096, 2048), (5504, 2048, 513)], **ids)
def test_weight_gradients_of_a_training_step(size):
    """Both gradients and one, by the library's plans for these sizes."""
    M, N, K = size
    gen = torch.Generator(device=DEV)
    gen.manual_seed(M)
    dg, du, x = (torch.randn(K, c, device=DEV, generator=gen).to(BF16) for c in (M, M, N))
    print(ffn.ffn_plan(ffn.FFN_OP_GATED_DW, M, N, K), ffn.ffn_plan(ffn.FFN_OP_DW, M, N, K), flush=True)
    for got, want in zip((*b.gated_linear_dw(dg, du, x), b.linear_dw(dg, x)), (dg, du, dg)):
        ref.assert_within(got, ref.dw(want, x, torch.float32))
