"""The block-scaled entry points on a machine without a GPU: the declared functions are
exported, and bad arguments are refused before any HIP call."""
import os
import re

import pytest

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import mx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "mx_mi355x.h")
BAD = b.GEMM_ERR_INVALID_VALUE
X, Q, S, C = 0x10000000, 0x20000000, 0x30000000, 0x40000000    # never dereferenced


def test_header_declares_what_the_binding_calls_and_the_library_exports():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    declared = sorted(set(re.findall(r"^\s*int\s+(mx_\w+)\s*\(", text, flags=re.M)))
    assert declared == sorted(mx.EXPORTED)
    for name in declared:
        assert hasattr(b.lib(), name), name


def test_helpers_are_reached_through_the_binding():
    assert b.linear_mx4 is mx.linear_mx4 and b.pack_mx8 is mx.pack_mx8 and b.MxMatrix is mx.MxMatrix
    with pytest.raises(AttributeError):
        b.no_such_helper


# rows, cols, bf16 matrix, ldx, codes, ldq, scales, lds (the order of the pack calls)
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("args", [
    (-1, 64, X, 64, Q, 64, S, 2),
    (4, -1, X, 64, Q, 64, S, 2),
    (4, 64, X, 63, Q, 64, S, 2),                # rows of X overlap
    (4, 64, X, 64, Q, 31, S, 2),                # rows of codes too short, for both widths
    (4, 65, X, 65, Q, 65, S, 2),                # three blocks to a row
    (4, 64, 0, 64, Q, 64, S, 2),
    (4, 64, X, 64, 0, 64, S, 2),
    (4, 64, X, 64, Q, 64, 0, 2),
    (4, 64, X + 1, 64, Q, 64, S, 2),            # not a bf16 address
    (4, 64, X, 64, X + 8, 64, S, 2),            # codes in X
    (4, 64, X, 64, Q, 64, X + 300, 2),          # scales in X
    (4, 64, X, 1 << 62, Q, 64, S, 2),           # a stride past 64-bit byte offsets
    (1 << 60, 64, X, 64, Q, 64, S, 2),
    (2, 64, X, -64, Q, 64, S, 2),
])
def test_conversions_refuse(bits, args):
    rows, cols, x, ldx, q, ldq, s, lds = args
    pack, unpack = (mx.mx_pack4, mx.mx_unpack4) if bits == 4 else (mx.mx_pack8, mx.mx_unpack8)
    assert pack(rows, cols, x, ldx, q, ldq, s, lds) == BAD
    assert unpack(rows, cols, q, ldq, s, lds, x, ldx) == BAD


@pytest.mark.parametrize("bits", [4, 8])
def test_packing_refuses_outputs_that_overlap(bits):
    assert (mx.mx_pack4 if bits == 4 else mx.mx_pack8)(4, 64, X, 64, Q, 64, Q + 100, 2) == BAD


@pytest.mark.parametrize("bits", [4, 8])
def test_empty_conversions_do_nothing(bits):
    pack, unpack = (mx.mx_pack4, mx.mx_unpack4) if bits == 4 else (mx.mx_pack8, mx.mx_unpack8)
    for rows, cols in ((0, 64), (4, 0), (0, 0)):
        assert pack(rows, cols, 0, 0, 0, 0, 0, 0) == b.GEMM_OK
        assert unpack(rows, cols, 0, 0, 0, 0, 0, 0) == b.GEMM_OK


# Per form: the product, the rows and columns of A and B for M = 4, N = 64, K = 96, and B's bits.
FORMS = [(mx.mx_gemm_bf16_mx4_f32_bt, (4, 96), (64, 96), 4, 4), (mx.mx_gemm_bf16_mx4_bf16_bt, (4, 96), (64, 96), 4, 2),
         (mx.mx_gemm_bf16_mx4_f32, (4, 96), (96, 64), 4, 4), (mx.mx_gemm_bf16_mx4_bf16, (4, 96), (96, 64), 4, 2),
         (mx.mx_gemm_bf16_mx8_f32_at, (96, 4), (96, 64), 8, 4), (mx.mx_gemm_bf16_mx8_bf16_at, (96, 4), (96, 64), 8, 2)]


def _good(a, bm, bits):
    return dict(M=4, N=64, K=96, A=X, lda=a[1], codes=Q, ldq=bm[1] * bits // 8, scales=S, lds=-(-bm[1] // 32), C=C, ldc=64)


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f[0].__name__)
def test_products_refuse(form):
    fn, a, bm, bits, esize = form
    good = _good(a, bm, bits)
    bad = [dict(M=-1), dict(N=-1), dict(K=-1), dict(A=0), dict(codes=0), dict(scales=0), dict(C=0),
           dict(lda=good["lda"] - 1), dict(ldq=good["ldq"] - 1), dict(lds=good["lds"] - 1), dict(ldc=63),
           dict(A=X + 1), dict(C=C + 1), dict(C=C + esize // 2), dict(C=X + 8), dict(C=Q), dict(C=S),
           dict(lda=1 << 61), dict(ldq=1 << 61), dict(ldc=1 << 61), dict(M=1 << 60), dict(N=1 << 60), dict(lda=-96)]
    for change in bad:
        if fn.__name__.endswith("_at") and change == dict(lda=good["lda"] - 1):
            assert good["lda"] == 4     # rows of At hold M elements
        assert fn(**{**good, **change}) == BAD, change


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f[0].__name__)
def test_products_without_results_do_nothing(form):
    fn, a, bm, bits, _ = form
    good = _good(a, bm, bits)
    assert fn(**{**good, "M": 0, "A": 0, "C": 0}) == b.GEMM_OK
    assert fn(**{**good, "N": 0, "C": 0}) == b.GEMM_OK


def test_helpers_refuse_what_is_not_theirs():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    q4 = mx.MxMatrix(torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2, dtype=torch.uint8), 64)
    with pytest.raises(TypeError):
        mx.pack_mx4(x.float())
    with pytest.raises(ValueError):
        mx.pack_mx8(x)                          # not on a GPU
    with pytest.raises(TypeError):
        mx.linear_mx4(x.float(), q4)
    with pytest.raises(ValueError):
        mx.linear_mx4(x[:, :32], q4)            # 32 against 64 columns
    with pytest.raises(ValueError):
        mx.linear_mx4(x, q4)                    # not on a GPU
    with pytest.raises(ValueError):
        mx.linear_mx4(x[0], q4)                 # no matrix


def test_plans_and_their_hook():
    for op in (mx.MX_OP_FORWARD, mx.MX_OP_INPUT_GRADIENT, mx.MX_OP_WEIGHT_GRADIENT):
        for M, N, K in ((1, 14336, 4096), (16, 4096, 14336), (77, 130, 1), (2048, 11008, 4096), (5, 5, 0)):
            plan = mx.mx_plan(op, M, N, K)
            assert plan["config"] >= 0 and plan["name"].startswith("mx_") and plan["split_k"] >= 1
            # The slices cover K, and none of them is empty.
            assert plan["split_k"] * plan["k_chunk"] >= K and (K == 0 or (plan["split_k"] - 1) * plan["k_chunk"] < K)
        assert mx.mx_plan(op, 0, 5, 5)["config"] == -1
        for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1)):
            with pytest.raises(b.GemmError):
                mx.mx_plan(op, *bad)
        with pytest.raises(b.GemmError) as e:
            mx.mx_plan(op, 1 << 31, 1, 1)
        assert e.value.status == b.GEMM_ERR_UNSUPPORTED
        config = mx.mx_plan(op, 300, 300, 3000)["config"]
        assert mx.mx_force_plan((op + 1) % 3, config) == BAD
        try:
            assert mx.mx_force_plan(op, config, 3) == b.GEMM_OK
            assert mx.mx_plan(op, 5, 5, 3000)["config"] == config and mx.mx_plan(op, 5, 5, 3000)["split_k"] == 3
        finally:
            assert mx.mx_force_plan(op) == b.GEMM_OK
    for bad in ((3, -1, 0), (-1, -1, 0), (0, 64, 0), (0, -2, 0), (0, -1, -1)):
        assert mx.mx_force_plan(*bad) == BAD
