"""Operands whose rows overlap (expanded tensors, overlapping views) never reach a kernel: the helpers
hand the library the strides that the tensors have, and the library refuses the ones shorter than a row."""
import pytest
import torch

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import mx

BAD = b.GEMM_ERR_INVALID_VALUE
X, Q, S, C = 0x10000000, 0x20000000, 0x30000000, 0x40000000    # never dereferenced


# ---- on the CPU: the stride that a helper passes on, and that the C ABI refuses it

@pytest.mark.parametrize("make,want", [
    (lambda: torch.zeros(1, 4096).expand(8, 4096), 0),
    (lambda: torch.zeros(8192).as_strided((5, 4096), (1024, 1)), 1024),
    (lambda: torch.zeros(1, 1).expand(8, 1), 0),
    (lambda: torch.zeros(8, 4096), 4096),
    (lambda: torch.zeros(8, 4096)[:, :33], 4096),
    (lambda: torch.zeros(8, 4096)[:, :1], 4096),
    (lambda: torch.zeros(4096).expand(1, 4096), 4096),          # one row: any stride
    (lambda: torch.zeros(1, 4096)[:, 5:38], 33),
    (lambda: torch.zeros(8, 0), 1),
    (lambda: torch.zeros(0, 8), 8),
])
def test_the_row_stride_is_the_tensors(make, want):
    x = make()
    assert mx._ld(x.stride(), *x.shape) == want


@pytest.mark.parametrize("ld", [0, 16, 63])
def test_the_entry_points_refuse_rows_that_overlap(ld):
    for pack, unpack, half in ((mx.mx_pack4, mx.mx_unpack4, 2), (mx.mx_pack8, mx.mx_unpack8, 1)):
        for args in ((X, ld, Q, 64, S, 2), (X, 64, Q, ld // half, S, 2), (X, 64, Q, 64, S, min(ld, 1))):
            assert pack(4, 64, *args) == BAD
            assert unpack(4, 64, *args[2:], *args[:2]) == BAD
    short = min(ld, 1)
    for fn, lda, ldq, bits in ((mx.mx_gemm_bf16_mx4_f32_bt, 64, 32, 4), (mx.mx_gemm_bf16_mx4_f32, 64, 32, 4),
                               (mx.mx_gemm_bf16_mx8_f32_at, 64, 64, 8)):
        bad = ld * bits // 8
        for strides in ((ld, ldq, 2, 64), (lda, bad, 2, 64), (lda, ldq, short, 64), (lda, ldq, 2, ld)):
            la, lq, ls, lc = strides
            assert fn(64, 64, 64, X, la, Q, lq, S, ls, C, lc) == BAD, strides


# ---- on the GPU: each helper refuses such a tensor in each place, before any launch

def expanded(x):
    return x[:1].expand(x.shape[0], -1)


def refusals():
    dev = torch.device("cuda:0")
    x = torch.ones(64, 96, dtype=torch.bfloat16, device=dev)
    W, X8 = b.pack_mx4(x), b.pack_mx8(x)
    dy = torch.ones(64, 64, dtype=torch.bfloat16, device=dev)
    flat = torch.ones(64 * 96, dtype=torch.bfloat16, device=dev)
    overlapping = flat.as_strided((64, 96), (48, 1))
    f32 = torch.zeros(1, 96, device=dev)

    def with_codes(Q):
        return mx.MxMatrix(expanded(Q.codes), Q.scales, Q.cols)

    def with_scales(Q):
        return mx.MxMatrix(Q.codes, expanded(Q.scales), Q.cols)

    for pack in (b.pack_mx4, b.pack_mx8):
        yield lambda pack=pack: pack(expanded(x))
        yield lambda pack=pack: pack(overlapping)
        yield lambda pack=pack: pack(expanded(x)[:, :1])
    for Q in (W, X8):
        yield lambda Q=Q: b.unpack_mx(with_codes(Q))
        yield lambda Q=Q: b.unpack_mx(with_scales(Q))
        yield lambda Q=Q: b.unpack_mx(Q, out=expanded(x))
    for fn, a, Q, width in ((b.linear_mx4, x, W, 64), (b.linear_mx4_dx, dy, W, 96), (b.linear_mx8_dw, dy, X8, 96)):
        rows = a.shape[0]
        yield lambda fn=fn, a=a, Q=Q: fn(expanded(a), Q)
        yield lambda fn=fn, a=a, Q=Q: fn(flat.as_strided(a.shape, (a.shape[1] - 1, 1)), Q)
        yield lambda fn=fn, a=a, Q=Q: fn(a, with_codes(Q))
        yield lambda fn=fn, a=a, Q=Q: fn(a, with_scales(Q))
        yield lambda fn=fn, a=a, Q=Q, rows=rows, width=width: fn(a, Q, out=f32[:, :width].expand(rows, -1))


@pytest.mark.gpu
def test_helpers_refuse_rows_that_overlap():
    n = 0
    for call in refusals():
        with pytest.raises(b.GemmError) as e:
            call()
        assert e.value.status == BAD
        n += 1
    assert n == 27
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_a_gradient_that_was_expanded_is_taken_as_a_copy():
    """The gradient of a sum over tokens, made contiguous, is an operand like any other; one row of it
    needs no copy."""
    dev = torch.device("cuda:0")
    g = torch.randn(1, 64, device=dev).to(torch.bfloat16)
    W = b.pack_mx4(torch.randn(64, 96, device=dev).to(torch.bfloat16))
    rows = b.linear_mx4_dx(g.expand(40, 64).contiguous(), W)
    assert torch.equal(rows, rows[:1].expand(40, -1))
    assert torch.equal(b.linear_mx4_dx(g.expand(1, 64), W), b.linear_mx4_dx(g, W))
