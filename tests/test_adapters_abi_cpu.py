"""The adapter entry points on a machine without a GPU: the declared functions are exported, and bad arguments are
refused before any HIP call."""
import os
import re

import pytest

from paper_2512_13282_amd import adapters as ad
from paper_2512_13282_amd import binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "adapters_mi355x.h")
BAD, UNSUPPORTED = b.GEMM_ERR_INVALID_VALUE, b.GEMM_ERR_UNSUPPORTED
X, W, Y, H, INDEX, A, B, SCALE, DH, DA, DB = (0x10000000 * (i + 1) for i in range(11))    # never dereferenced
M, N, K, n, r = 4, 64, 96, 3, 8


def test_header_declares_what_the_binding_calls_and_the_library_exports():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"^\s*int\s+(adapters_\w+)\s*\(", text, flags=re.M))) == sorted(ad.EXPORTED)
    for name in ad.EXPORTED:
        assert hasattr(b.lib(), name), name


def test_helpers_are_reached_through_the_binding():
    assert b.linear_adapters is ad.linear_adapters and b.Adapters is ad.Adapters


def linear(fn, forward, held=True, **change):
    n_out, n_in = (N, K) if forward else (K, N)
    s = dict(n=n, r=r, A=A, lda=n_in, sa=r * n_in, B=B, ldb=r, sb=n_out * r, scale=SCALE)
    a = dict(M=M, N=N, K=K, X=X, ldx=K, W=W, ldw=n_in, index=INDEX, Y=Y, ldy=N, H=H)
    for k, v in change.items():
        (s if k in s else a)[k] = v
    held = ad.AdaptersSet(s["n"], s["r"], s["A"] or None, s["lda"], s["sa"], s["B"] or None, s["ldb"], s["sb"], s["scale"] or None) if held else None
    return fn(a["M"], a["N"], a["K"], a["X"], a["ldx"], a["W"], a["ldw"], held, a["index"], a["Y"], a["ldy"], a["H"])


FORMS = [(ad.adapters_linear_f32_bt, True, 4), (ad.adapters_linear_bf16_bt, True, 2), (ad.adapters_linear_f32, False, 4),
         (ad.adapters_linear_bf16, False, 2)]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f[0].__name__)
def test_products_refuse(form):
    fn, forward, size = form
    n_out, n_in = (N, K) if forward else (K, N)
    bad = [dict(held=False), dict(M=-1), dict(N=-1), dict(K=-1), dict(n=-1), dict(r=-1), dict(X=0), dict(W=0), dict(Y=0), dict(A=0), dict(B=0),
           dict(index=0), dict(ldx=K - 1), dict(ldw=n_in - 1), dict(ldy=N - 1), dict(lda=n_in - 1), dict(ldb=r - 1), dict(X=X + 1), dict(W=W + 1),
           dict(A=A + 1), dict(B=B + 1), dict(Y=Y + size // 2), dict(H=H + 2), dict(index=INDEX + 2), dict(scale=SCALE + 2),
           dict(sa=r * n_in - 1), dict(sb=n_out * r - 1), dict(sa=0), dict(sb=-5), dict(sa=1 << 60), dict(lda=1 << 60), dict(ldx=1 << 60),
           dict(n=1 << 50), dict(M=1 << 60)]
    for place in (X, W, A, B, INDEX, SCALE):
        bad += [dict(Y=place), dict(H=place)]
    bad += [dict(Y=H), dict(Y=A + 2 * 2 * r * n_in), dict(H=B + 4)]
    for change in bad:
        assert linear(fn, forward, **change) == BAD, change
    assert linear(fn, forward, M=0) == b.GEMM_OK
    assert linear(fn, forward, N=0, H=0) == b.GEMM_OK
    assert linear(fn, forward, M=0, X=0, W=W, index=0, Y=0, H=0) == b.GEMM_OK


@pytest.mark.parametrize("form", FORMS, ids=lambda f: f[0].__name__)
def test_what_no_kernel_takes_is_unsupported(form):
    fn, forward, _ = form
    far = dict(X=1 << 44, W=2 << 44, Y=3 << 44, H=4 << 44, A=5 << 44, B=6 << 44, index=7 << 44, scale=8 << 44)
    assert linear(fn, forward, **far, r=2000, ldb=2000, sa=2000 * 96, sb=2000 * 96) == UNSUPPORTED
    assert linear(fn, forward, **far, M=(1 << 26) + 1) == UNSUPPORTED
    k = 1 << 31
    assert linear(fn, forward, **far, K=k, ldx=k, ldw=k if forward else N, lda=k if forward else N, sa=8 * k if forward else 8 * N, sb=8 * k) == UNSUPPORTED


def gradients(fn, **change):
    a = dict(M=M, N=N, K=K, n=n, r=r, X=X, ldx=K, dY=Y, lddy=N, H=H, dH=DH, index=INDEX, dA=DA, ldda=K, sda=r * K, dB=DB, lddb=r, sdb=N * r)
    a.update(change)
    return fn(*a.values())


@pytest.mark.parametrize("fn,size", [(ad.adapters_dw_f32, 4), (ad.adapters_dw_bf16, 2)], ids=["f32", "bf16"])
def test_weight_gradients_refuse(fn, size):
    bad = [dict(M=-1), dict(N=-1), dict(K=-1), dict(n=-1), dict(r=-1), dict(X=0), dict(dY=0), dict(H=0), dict(dH=0), dict(index=0), dict(dA=0), dict(dB=0),
           dict(ldx=K - 1), dict(lddy=N - 1), dict(ldda=K - 1), dict(lddb=r - 1), dict(sda=r * K - 1), dict(sdb=N * r - 1), dict(X=X + 1), dict(H=H + 2),
           dict(dH=DH + 2), dict(index=INDEX + 2), dict(dA=DA + size // 2), dict(dB=DB + size // 2), dict(dB=DA + size * 8), dict(sda=1 << 60), dict(M=1 << 60)]
    for place in (X, Y, H, DH, INDEX):
        bad += [dict(dA=place), dict(dB=place)]
    for change in bad:
        assert gradients(fn, **change) == BAD, change
    far = dict(X=1 << 50, dY=2 << 50, H=3 << 50, dH=4 << 50, index=5 << 50, dA=6 << 50, dB=7 << 50)
    assert gradients(fn, **far, n=65536) == UNSUPPORTED
    assert gradients(fn, **far, r=2000, lddb=2000, sda=2000 * K, sdb=2000 * N) == UNSUPPORTED
    assert gradients(fn, **far, K=1 << 30, ldx=1 << 30, ldda=1 << 30, sda=8 << 30) == UNSUPPORTED
    assert gradients(fn, n=0) == b.GEMM_OK and gradients(fn, r=0) == b.GEMM_OK and gradients(fn, N=0, K=0) == b.GEMM_OK


def test_the_plan_hook():
    for op in (0, 1):
        assert ad.adapters_force_plan(op, 0, 2) == b.GEMM_OK and ad.adapters_force_plan(op) == b.GEMM_OK
    for bad in ((2, -1, 0), (-1, -1, 0), (0, 64, 0), (0, -2, 0), (0, -1, -1)):
        assert ad.adapters_force_plan(*bad) == BAD


def test_helpers_refuse_what_is_not_theirs():
    torch = pytest.importorskip("torch")
    bf16 = torch.bfloat16
    x, w, index = torch.zeros(4, 96, dtype=bf16), torch.zeros(64, 96, dtype=bf16), torch.zeros(4, dtype=torch.int32)
    held = b.Adapters(torch.zeros(3, 8, 96, dtype=bf16), torch.zeros(3, 64, 8, dtype=bf16))
    with pytest.raises(TypeError):
        b.linear_adapters(x.float(), w, held, index)
    with pytest.raises(ValueError):
        b.linear_adapters(x, w, held, index)             # not on a GPU
    with pytest.raises(ValueError):
        b.linear_adapters_dw(x, x, torch.zeros(4, 8), torch.zeros(4, 8), index, 3)


def test_negative_strides_past_64_bits_of_bytes_are_refused():
    """A stride whose bytes wrap round to a large positive number."""
    far = lambda size: -(1 << 64) // size + (1 << 30)        # noqa: E731
    for fn, forward, size in FORMS:
        for k, v in (("ldx", far(2)), ("ldw", far(2)), ("lda", far(2)), ("ldb", far(2)), ("sa", far(2)), ("sb", far(2)), ("ldy", far(size))):
            assert linear(fn, forward, **{k: v}) == BAD, (fn.__name__, k)
    for fn, size in ((ad.adapters_dw_f32, 4), (ad.adapters_dw_bf16, 2)):
        for k, v in (("ldx", far(2)), ("lddy", far(2)), ("ldda", far(size)), ("lddb", far(size)), ("sda", far(size)), ("sdb", far(size))):
            assert gradients(fn, **{k: v}) == BAD, (fn.__name__, k)
