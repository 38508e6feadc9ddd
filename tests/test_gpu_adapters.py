"""The projection with adapters against its definition in 64 bits, within the bounds of its fp32 sums and its one
rounding (fused_reference.py)."""
import pytest
import torch

import fused_reference as ref
from paper_2512_13282_amd import adapters as ad
from paper_2512_13282_amd import binding as b
from test_gpu_ffn import BF16, DEV, generator, ids, leaves_rows, matrix

pytestmark = pytest.mark.gpu

# M, N, K, adapters, rank, pad, offset
SIZES = [(1, 8, 8, 1, 8, 0, 0), (1, 1, 1, 1, 1, 0, 0), (3, 7, 5, 2, 3, 0, 0), (16, 128, 256, 16, 16, 0, 0), (37, 131, 129, 5, 7, 1, 3),
         (64, 256, 520, 3, 16, 8, 8), (65, 130, 1000, 70, 4, 0, 0), (130, 264, 320, 1, 64, 0, 0), (300, 513, 511, 9, 33, 5, 1),
         (257, 520, 136, 4, 128, 0, 0), (1, 1000, 2056, 3, 16, 0, 0), (12, 512, 4104, 40, 32, 0, 0), (511, 264, 64, 2, 1, 0, 0), (40, 96, 200, 2, 300, 0, 0),
         # More tiles than compute units: whole ones, and slices of the rest.
         (1100, 4200, 200, 6, 16, 0, 0), (4340, 4100, 264, 7, 24, 0, 4)]


def indices(gen, M, n):
    """An adapter a token: requests one after the other, and in no order with tokens that have none."""
    cuts = torch.sort(torch.randint(0, M + 1, (max(n - 1, 0),), generator=gen)).values
    yield "in order", torch.bucketize(torch.arange(M), cuts, right=True).clamp(max=n - 1).to(torch.int32)
    none = torch.tensor([-1, n, -(1 << 31), (1 << 31) - 1])
    mixed = torch.where(torch.rand(M, generator=gen) < 0.2, none[torch.randint(0, 4, (M,), generator=gen)], torch.randint(0, n, (M,), generator=gen))
    yield "mixed", mixed.to(torch.int32)


def stacked(gen, n, rows, cols, scale, pad, offset):
    """n matrices in a buffer of NaN, rows `pad` apart and the matrices 3 more rows."""
    flat = matrix(gen, n * (rows + 3), cols, scale, pad, offset)
    return flat.as_strided((n, rows, cols), ((rows + 3) * (cols + pad), cols + pad, 1))


def configurations(op):
    found = [c for c in range(64) if ad.adapters_force_plan(op, c) == b.GEMM_OK]
    ad.adapters_force_plan(op)
    return found


def plans(op, call):
    """The library's plan, then every configuration with one slice and three."""
    yield "own", call()
    try:
        for config in configurations(op):
            for split in (1, 3):
                assert ad.adapters_force_plan(op, config, split) == b.GEMM_OK
                try:
                    got = call()
                except b.GemmError as e:
                    assert e.status == b.GEMM_ERR_UNSUPPORTED
                    continue
                yield (config, split), got
    finally:
        ad.adapters_force_plan(op)


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, **ids)
@pytest.mark.parametrize("forward", [True, False], ids=["fwd", "dx"])
def test_linear(forward, size, dtype):
    M, N, K, n, r, pad, offset = size
    gen = generator("linear", forward, *size)
    n_out, n_in = (N, K) if forward else (K, N)
    x, w = matrix(gen, M, K, 1.0, pad, offset), matrix(gen, n_out, n_in, K ** -0.5, pad, offset)
    A, B = stacked(gen, n, r, n_in, K ** -0.5, pad, offset), stacked(gen, n, n_out, r, 1.0, pad, offset)
    for scale in (None, (torch.rand(n, generator=gen) + 0.5).to(DEV)):
        for what, index in indices(gen, M, n):
            held = ad.Adapters(A, B, scale)
            at = index.to(DEV)
            if forward:
                call = lambda: b.linear_adapters(x, w, held, at, out_dtype=dtype, keep=True)       # noqa: E731
                want = ref.adapted(x, w.t(), A.transpose(1, 2), B.transpose(1, 2), scale, index, dtype)
            else:
                call = lambda: b.linear_adapters_dx(x, w, held, at, out_dtype=dtype, keep=True)    # noqa: E731
                want = ref.adapted(x, w, B, A, scale, index, dtype)
            print(forward, size, what, flush=True)
            for plan, (y, h) in plans(0 if forward else 1, call):
                ref.assert_within(h, want[1], f"h {what} {plan}")
                ref.assert_within(y, want[0], f"y {what} {plan}")
            fn = b.linear_adapters if forward else b.linear_adapters_dx
            assert torch.equal(fn(x, w, held, at, out_dtype=dtype), call()[0])


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, **ids)
def test_weight_gradients(size, dtype):
    M, N, K, n, r, pad, offset = size
    gen = generator("dw", *size)
    x, dy = matrix(gen, M, K, 1.0, pad, offset), matrix(gen, M, N, 1.0, pad, offset)
    h, dh = torch.randn(M, r, generator=gen).to(DEV), torch.randn(M, r, generator=gen).to(DEV)
    for what, index in indices(gen, M, n):
        print(size, what, flush=True)
        got = b.linear_adapters_dw(x, dy, h, dh, index.to(DEV), n, out_dtype=dtype)
        for g, w, name in zip(got, ref.adapter_dw(x, dy, h, dh, index, n, dtype), ("dA", "dB")):
            ref.assert_within(g, w, f"{name} {what}")


def test_an_adapter_reaches_its_own_tokens_only():
    """NaN and infinities in one request's adapter, activations and h: the other rows and adapters keep their bits."""
    gen = generator("isolation")
    M, N, K, n, r = 96, 200, 136, 4, 20
    x, w = matrix(gen, M, K), matrix(gen, N, K)
    A, B = stacked(gen, n, r, K, 0.1, 0, 0), stacked(gen, n, N, r, 0.1, 0, 0)
    index = torch.randint(-1, n, (M,), generator=gen).to(torch.int32)
    at, other = index.to(DEV), (index != 2).to(DEV)
    y, h = b.linear_adapters(x, w, ad.Adapters(A, B), at, keep=True)
    v = matrix(gen, K, N)
    A2, B2 = stacked(gen, n, r, N, 0.1, 0, 0), stacked(gen, n, K, r, 0.1, 0, 0)
    dx, dh = b.linear_adapters_dx(x, v, ad.Adapters(A2, B2), at, keep=True)
    dA, dB = b.linear_adapters_dw(x, y, h, dh, at, n)
    for bad in (float("nan"), float("inf")):
        for t in (A, B, A2, B2):
            t[2] = bad
        y2, h2 = b.linear_adapters(x, w, ad.Adapters(A, B), at, keep=True)
        assert torch.equal(y2[other], y[other]) and torch.equal(h2[other], h[other])
        assert not torch.any(torch.isfinite(h2[~other])) and not torch.any(torch.isfinite(y2[~other]))
        dx2, dh2 = b.linear_adapters_dx(x, v, ad.Adapters(A2, B2), at, keep=True)
        assert torch.equal(dx2[other], dx[other]) and torch.equal(dh2[other], dh[other])
        dA2, dB2 = b.linear_adapters_dw(x, y2, h2, dh2, at, n)
        for i in (0, 1, 3):
            assert torch.equal(dA2[i], dA[i]) and torch.equal(dB2[i], dB[i])


def test_values_at_the_ends_of_their_range():
    """An h of one large and many small values keeps its 24 bits into an fp32 result; an infinite h stays infinite."""
    K, N, r = 8, 32, 24
    x = torch.zeros(2, K, dtype=BF16, device=DEV)
    x[0, 0] = 1
    A, B = torch.zeros(1, r, K, dtype=BF16, device=DEV), torch.zeros(1, N, r, dtype=BF16, device=DEV)
    A[0, :, 0] = torch.tensor([1 + i / 128 for i in range(r)])
    B[0, :, 3] = 1
    B[0, :, 23] = 2.0 ** -9
    scale = torch.tensor([1.0000001], device=DEV)
    w = torch.zeros(N, K, dtype=BF16, device=DEV)
    index = torch.zeros(2, dtype=torch.int32, device=DEV)
    y = b.linear_adapters(x, w, ad.Adapters(A, B, scale), index, out_dtype=torch.float32)
    s = scale.double()
    want = (1 + 3 / 128) * s + 2.0 ** -9 * (1 + 23 / 128) * s
    assert torch.all((y[0].double() - want).abs() <= 4 * 2.0 ** -23) and torch.all(y[1] == 0)
    A[0, 3, 0] = float("inf")
    B[0, :, 23] = 0
    y = b.linear_adapters(x, w, ad.Adapters(A, B, scale), index)
    assert torch.all(torch.isnan(y[1]) | (y[1] == 0))          # 0 times the infinity is a NaN of its own row
    x[1, 0] = 1
    y, h = b.linear_adapters(x, w, ad.Adapters(A, B[:, :, 3:4].contiguous().expand(1, N, r).contiguous(), scale), index, keep=True)
    assert torch.all(h[:, 3] == float("inf")) and torch.all(y == float("inf"))


def test_no_adapters_and_no_rank_are_the_projection_alone():
    gen = generator("none")
    x, w = matrix(gen, 40, 96), matrix(gen, 72, 96)
    index = torch.zeros(40, dtype=torch.int32, device=DEV)
    e = lambda *s: torch.empty(*s, dtype=BF16, device=DEV)          # noqa: E731
    want = ref.product(x, w.t())
    for n, r in ((0, 16), (3, 0), (0, 0)):
        y, h = b.linear_adapters(x, w, ad.Adapters(e(n, r, 96), e(n, 72, r)), index, out_dtype=torch.float32, keep=True)
        ref.assert_within(y, want)
        assert h.shape == (40, r) and (n > 0 or r == 0 or torch.all(h == 0))
        dA, dB = b.linear_adapters_dw(x, y.to(BF16), h, h, index, n)
        assert dA.shape == (n, r, 96) and dB.shape == (n, 72, r)
    A, B = matrix(gen, 3 * 8, 96).view(3, 8, 96), matrix(gen, 3 * 72, 8).view(3, 72, 8)
    none = torch.full((40,), -1, dtype=torch.int32, device=DEV)
    y, h = b.linear_adapters(x, w, ad.Adapters(A, B), none, out_dtype=torch.float32, keep=True)
    ref.assert_within(y, want)
    assert torch.all(h == 0)
    dA, dB = b.linear_adapters_dw(x, y.to(BF16), h + 1, h + 1, none, 3)
    assert torch.all(dA == 0) and torch.all(dB == 0)
    # No tokens, no inputs, no outputs.
    dA, dB = b.linear_adapters_dw(x[:0], y[:0].to(BF16), h[:0], h[:0], none[:0], 3)
    assert torch.all(dA == 0) and torch.all(dB == 0)
    assert b.linear_adapters(x[:0], w, ad.Adapters(A, B), none[:0]).shape == (0, 72)
    y, h = b.linear_adapters(e(40, 0), e(72, 0), ad.Adapters(e(3, 8, 0), B), index, keep=True)
    assert torch.all(y == 0) and torch.all(h == 0)
    y, h = b.linear_adapters(x, w[:0], ad.Adapters(A, e(3, 0, 8)), index, keep=True)
    assert y.shape == (40, 0)
    ref.assert_within(h, ref.adapted(x, w.t(), A.transpose(1, 2), B.transpose(1, 2), None, index, BF16)[1])


@pytest.mark.parametrize("tokens", [1, 7, 90])
def test_captured_calls_read_the_index_and_the_adapters_anew(tokens):
    gen = generator("capture", tokens)
    N, K, n, r = 200, 1032, 5, 16
    x, w = matrix(gen, tokens, K), matrix(gen, N, K)
    A, B = stacked(gen, n, r, K, 0.1, 0, 0), stacked(gen, n, N, r, 0.1, 0, 0)
    scale = torch.ones(n, device=DEV)
    index = torch.zeros(tokens, dtype=torch.int32, device=DEV)
    held = ad.Adapters(A, B, scale)

    def step():
        y, h = b.linear_adapters(x, w, held, index, keep=True)
        dx, dh = b.linear_adapters_dx(y, w, held, index, keep=True)
        return y, h, dx, dh, *b.linear_adapters_dw(x, y, h, dh, index, n)

    for split in (0, 3):
        for op in (0, 1):
            assert ad.adapters_force_plan(op, -1, split) == b.GEMM_OK
        try:
            torch.cuda.synchronize()
            assert b.gemm_release_workspace() == b.GEMM_OK
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
                kept = step()
            for _ in range(3):
                index.copy_(torch.randint(-1, n, (tokens,), generator=gen))
                scale.uniform_(0.5, 1.5)
                A.normal_(std=0.1)
                x.normal_()
                want = step()
                for t in kept:
                    t.fill_(7.0)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                for a, c in zip(kept, want):
                    assert torch.equal(a, c)
            del graph
        finally:
            for op in (0, 1):
                ad.adapters_force_plan(op)
    torch.cuda.synchronize()
    assert b.gemm_release_workspace() == b.GEMM_OK


def test_results_leave_their_padding():
    gen = generator("padding")
    x, w = matrix(gen, 70, 96), matrix(gen, 133, 96)
    A, B = stacked(gen, 2, 5, 96, 0.1, 0, 0), stacked(gen, 2, 133, 5, 0.1, 0, 0)
    index = torch.randint(-1, 2, (70,), generator=gen).to(torch.int32).to(DEV)
    for dtype in (torch.float32, BF16):
        buf = torch.full((70, 140), 7.0, dtype=dtype, device=DEV)
        b.linear_adapters(x, w, ad.Adapters(A, B), index, out=buf[:, :133])
        assert torch.equal(buf[:, :133], b.linear_adapters(x, w, ad.Adapters(A, B), index, out_dtype=dtype)) and torch.all(buf[:, 133:] == 7)
    # Gradients into slices of larger stacks, by the entry point.
    h = torch.randn(70, 5, device=DEV)
    y = buf[:, :133]
    want = b.linear_adapters_dw(x, y, h, h, index, 2)
    dA, dB = torch.full((2, 6, 100), 7.0, device=DEV), torch.full((2, 140, 9), 7.0, device=DEV)
    rc = ad.adapters_dw_f32(70, 133, 96, 2, 5, x.data_ptr(), 96, y.data_ptr(), 140, h.data_ptr(), h.data_ptr(), index.data_ptr(), dA.data_ptr(),
                            100, 600, dB.data_ptr(), 9, 1260, torch.cuda.current_stream().cuda_stream)
    assert rc == b.GEMM_OK
    assert torch.equal(dA[:, :5, :96], want[0]) and torch.equal(dB[:, :133, :5], want[1])
    assert torch.all(dA[:, 5:] == 7) and torch.all(dA[:, :, 96:] == 7) and torch.all(dB[:, 133:] == 7) and torch.all(dB[:, :, 5:] == 7)


@pytest.mark.parametrize("none", [range(0, 40), range(64, 128), range(96, 300), range(0, 1)])
def test_rows_without_an_adapter_beside_one_of_nan(none):
    """Rows that share a tile with one adapter's rows and have none keep their bits whatever the adapter holds."""
    gen = generator("none beside", none.start, none.stop)
    M, N, K, r = 300, 270, 136, 20
    x, w, v = matrix(gen, M, K), matrix(gen, N, K), matrix(gen, K, N)
    index = torch.zeros(M, dtype=torch.int32)
    index[list(none)] = -1
    rows, index = (index < 0).to(DEV), index.to(DEV)
    bad = torch.full((1, r, max(N, K)), float("nan"), dtype=BF16, device=DEV)
    for op, fn, weight, n_in, n_out in ((0, b.linear_adapters, w, K, N), (1, b.linear_adapters_dx, v, N, K)):
        held = ad.Adapters(bad[:, :, :n_in], bad[:, :, :n_out].transpose(1, 2).contiguous())
        for plan, y in plans(op, lambda: fn(x, weight, held, index)):
            assert torch.all(torch.isfinite(y[rows])) and torch.all(torch.isnan(y[~rows])), plan


def test_adapters_past_four_gib():
    """Many adapters of a wide projection: the last one's matrices lie past 32-bit offsets."""
    gen = generator("large")
    n, r, N, K = 700, 64, 50000, 72
    x, w = matrix(gen, 33, K), matrix(gen, N, K)
    A = torch.zeros(n, r, K, dtype=BF16, device=DEV)
    B = torch.zeros(n, N, r, dtype=BF16, device=DEV)               # 4.5 GB
    A[-1].normal_(std=0.1)
    B[-1].normal_(std=0.1)
    index = torch.full((33,), n - 1, dtype=torch.int32)
    index[5] = 3
    at = index.to(DEV)
    alone = ad.Adapters(A[-1:].clone(), B[-1:].clone())
    one = torch.where(at == n - 1, 0, -1).to(torch.int32)
    y, h = b.linear_adapters(x, w, ad.Adapters(A, B), at, keep=True)
    y1, h1 = b.linear_adapters(x, w, alone, one, keep=True)
    assert torch.equal(h, h1) and torch.equal(y, y1)
    dA, dB = b.linear_adapters_dw(x, y, h, h, at, n)
    dA1, dB1 = b.linear_adapters_dw(x, y, h, h, one, 1)
    assert torch.equal(dA[-1], dA1[0]) and torch.equal(dB[-1], dB1[0]) and torch.all(dB[3] == 0) and torch.all(dB[n - 2] == 0)
    v = matrix(gen, N, 24)                                          # input gradient over the same B, N outputs
    A2 = matrix(gen, r, 24).view(1, r, 24).expand(n, r, 24).contiguous()
    dx = b.linear_adapters_dx(y, v, ad.Adapters(A2, B), at, out_dtype=torch.float32)
    dx1 = b.linear_adapters_dx(y, v, ad.Adapters(A2[:1].contiguous(), alone.B), one, out_dtype=torch.float32)
    assert torch.equal(dx[index != 3], dx1[index != 3])


def matches(got, terms, what):
    """What is not finite of the sums over terms' second axis (fp64, on the CPU), and nothing else."""
    want = terms.sum(1)
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got == float("inf"), want == float("inf")) and torch.equal(got == -float("inf"), want == -float("inf")), what


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("M", [12, 40, 300])
@pytest.mark.parametrize("one", [True, False], ids=["one adapter", "several"])
def test_infinities_are_what_the_formula_makes_of_them(M, one, dtype):
    """An infinity times an h of either sign is one whatever the bits of h: exact in bf16 (every other token), to 24 bits, or 0."""
    gen = generator("infinities", M, one)
    N, K, n, r = 72, 64, 3, 5
    index = torch.zeros(M, dtype=torch.int32) if one else torch.randint(0, n, (M,), generator=gen).to(torch.int32)
    at = index.to(DEV)
    x = matrix(gen, M, K)
    x[::2] = 0
    x[torch.arange(0, M, 2), torch.randint(0, K, ((M + 1) // 2,), generator=gen)] = 1.0
    down = matrix(gen, n * r, K).view(n, r, K)
    down[:, 2, :20] = 0                                             # an h of 0
    up = matrix(gen, n * N, r).view(n, N, r)
    for i in range(n):
        up[i, 3 + i, 0] = float("inf")
        up[i, 20, 1], up[i, 21, 2], up[i, 22, 3] = -float("inf"), float("inf"), float("nan")
        up[i, 70, 0], up[i, 70, 4] = float("inf"), -float("inf")
    w, v = matrix(gen, N, K), matrix(gen, K, N)
    for op, call in ((0, lambda: b.linear_adapters(x, w, ad.Adapters(down, up), at, out_dtype=dtype, keep=True)),
                     (1, lambda: b.linear_adapters_dx(x, v, ad.Adapters(up.transpose(1, 2).contiguous(), down.transpose(1, 2).contiguous()), at,
                                                      out_dtype=dtype, keep=True))):
        for plan, (y, h) in plans(op, call):
            assert torch.all(torch.isfinite(h))
            matches(y, h.double().cpu()[:, :, None] * up.double().cpu()[index.long()].transpose(1, 2), (op, plan))


@pytest.mark.parametrize("dtype", [torch.float32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("r", [5, 20, 70])
def test_infinities_of_the_activations_in_the_weight_gradients(r, dtype):
    gen = generator("infinities dw", r)
    M, N, K, n = 150, 72, 100, 3
    index = torch.randint(0, n, (M,), generator=gen).to(torch.int32)
    x, dy = matrix(gen, M, K), matrix(gen, M, N)
    h, dh = torch.randn(M, r, generator=gen), torch.randn(M, r, generator=gen)
    h[::2], dh[::2] = h[::2].to(BF16).float(), dh[::2].to(BF16).float()
    h[4, 1], dh[4, 1] = 0.0, 0.0
    for z, cols in ((x, K), (dy, N)):
        z[4, 7], z[5, 8], z[20, 9], z[21, cols - 1] = float("inf"), -float("inf"), float("nan"), float("inf")
        z[30, 40], z[31, 40] = float("inf"), -float("inf")
    dA, dB = b.linear_adapters_dw(x, dy, h.to(DEV), dh.to(DEV), index.to(DEV), n, out_dtype=dtype)
    for i in range(n):
        t = torch.nonzero(index == i)[:, 0]
        matches(dA[i], dh.double()[t].t()[:, :, None] * x.double().cpu()[t][None], ("dA", i))
        matches(dB[i].t(), h.double()[t].t()[:, :, None] * dy.double().cpu()[t][None], ("dB", i))


@pytest.mark.parametrize("config", [4, 5])
@pytest.mark.parametrize("op", [0, 1])
def test_lower_tiles_over_the_last_rows(op, config):
    """Whole rounds of 256 x 256 tiles over all columns, then lower tiles over the last rows, each row with its adapter."""
    gen = generator("row tails", op)
    M, N, K, n, r = 22950, 651, 40, 3, 5
    n_out, n_in = (N, K) if op == 0 else (K, N)
    x, w = matrix(gen, M, K), matrix(gen, n_out, n_in, K ** -0.5)
    A, B = stacked(gen, n, r, n_in, K ** -0.5, 0, 0), stacked(gen, n, n_out, r, 1.0, 0, 0)
    index = torch.randint(-1, n, (M,), generator=gen).to(torch.int32)
    at = index.to(DEV)
    assert leaves_rows(M, N, 1)
    try:
        assert ad.adapters_force_plan(op, config, 1) == b.GEMM_OK
        y = (b.linear_adapters if op == 0 else b.linear_adapters_dx)(x, w, ad.Adapters(A, B), at)
    finally:
        ad.adapters_force_plan(op)
    down, up = (A.transpose(1, 2), B.transpose(1, 2)) if op == 0 else (B, A)
    ref.assert_within(y, ref.adapted(x, w.t() if op == 0 else w, down, up, None, index, BF16)[0])
