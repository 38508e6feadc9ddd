"""The feed-forward entry points on a machine without a GPU: the declared functions are exported, and bad
arguments are refused before any HIP call."""
import os
import re

import pytest

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import ffn

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ffn_mi355x.h")
BAD, UNSUPPORTED = b.GEMM_ERR_INVALID_VALUE, b.GEMM_ERR_UNSUPPORTED
AT = [0x10000000 * (i + 1) for i in range(10)]           # never dereferenced


def test_header_declares_what_the_binding_calls_and_the_library_exports():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"^\s*int\s+(ffn_\w+)\s*\(", text, flags=re.M))) == sorted(ffn.EXPORTED)
    for name in ffn.EXPORTED:
        assert hasattr(b.lib(), name), name
    values = dict(re.findall(r"FFN_(\w+) = (\d)", text))
    assert {k: int(values[k.upper()]) for k in ffn.ACTIVATIONS} == ffn.ACTIVATIONS


def test_helpers_are_reached_through_the_binding():
    assert b.gated_linear is ffn.gated_linear and b.linear_dw is ffn.linear_dw
    with pytest.raises(AttributeError):
        b.no_such_helper


# M = 4, N = 64, K = 96.  Per form: the entry point, its operands and results as (rows, cols, element size) in the
# order of the call, and how many of them are operands.
M, N, K = 4, 64, 96
FORMS = {
    "gated": (ffn.ffn_gated_bf16_bt, [(M, K, 2), (N, K, 2), (N, K, 2), "act", (M, N, 2), (M, N, 2), (M, N, 2)], 3),
    "grad": (ffn.ffn_gated_grad_bf16, [(M, K, 2), (K, N, 2), (M, N, 2), (M, N, 2), "act", (M, N, 2), (M, N, 2), (M, N, 2)], 4),
    "dx_f32": (ffn.ffn_gated_dx_f32, [(M, K, 2), (K, N, 2), (M, K, 2), (K, N, 2), (M, N, 4)], 4),
    "dx_bf16": (ffn.ffn_gated_dx_bf16, [(M, K, 2), (K, N, 2), (M, K, 2), (K, N, 2), (M, N, 2)], 4),
    "gated_dw_f32": (ffn.ffn_gated_dw_f32, [(K, M, 2), (K, M, 2), (K, N, 2), (M, N, 4), (M, N, 4)], 3),
    "gated_dw_bf16": (ffn.ffn_gated_dw_bf16, [(K, M, 2), (K, M, 2), (K, N, 2), (M, N, 2), (M, N, 2)], 3),
    "dw_f32": (ffn.ffn_dw_f32, [(K, M, 2), (K, N, 2), (M, N, 4)], 2),
    "dw_bf16": (ffn.ffn_dw_bf16, [(K, M, 2), (K, N, 2), (M, N, 2)], 2),
}


def arguments(form, sizes=(M, N, K), act=0, change=None):
    """The call's arguments; change: (which matrix, address or None, row stride or None)."""
    fn, parts, operands = FORMS[form]
    args, i = list(sizes), 0
    for part in parts:
        if part == "act":
            args.append(act)
            continue
        p, ld = AT[i], part[1]
        if change is not None and change[0] == i:
            p, ld = (p if change[1] is None else change[1]), (ld if change[2] is None else change[2])
        args += [p, ld]
        i += 1
    return fn, args


def test_the_gradients_from_that_of_h_refuse():
    good = [M, N, AT[0], N, AT[1], N, AT[2], N, 0, AT[3], N, AT[4], N]
    bad = [(0, -1), (1, -1), (0, 1 << 60), (8, 4), (8, -1)]
    bad += [(i, v) for i in (2, 4, 6, 9, 11) for v in (0, good[i] + 1)] + [(i, v) for i in (3, 5, 7, 10, 12) for v in (N - 1, -N, 1 << 61)]
    bad += [(o, AT[i]) for o in (9, 11) for i in range(3)] + [(11, AT[3] + 4)]
    for i, v in bad:
        args = list(good)
        args[i] = v
        assert ffn.ffn_gated_bwd_bf16(*args) == BAD, (i, v)
    assert ffn.ffn_gated_bwd_bf16(0, N, *good[2:]) == b.GEMM_OK and ffn.ffn_gated_bwd_bf16(M, 0, *good[2:]) == b.GEMM_OK


@pytest.mark.parametrize("form", FORMS)
def test_refusals(form):
    fn, parts, operands = FORMS[form]
    matrices = [p for p in parts if p != "act"]

    def refused(**kw):
        f, args = arguments(form, **kw)
        assert f(*args) == BAD, kw

    for i in range(3):
        refused(sizes=tuple(-1 if j == i else s for j, s in enumerate((M, N, K))))
    for i in range(2):
        refused(sizes=tuple(1 << 60 if j == i else s for j, s in enumerate((M, N, K))))
    for i, (rows, cols, size) in enumerate(matrices):
        optional = (form == "grad" and i == 6)
        if not optional:
            refused(change=(i, 0, None))
        refused(change=(i, AT[i] + size // 2, None))
        refused(change=(i, None, cols - 1))
        refused(change=(i, None, -cols))
        refused(change=(i, None, 1 << 61))
        for o in range(operands, len(matrices)):             # a result in an operand or in another result
            if i < o:
                refused(change=(o, AT[i] + 8 * size, None))
    if "act" in parts:
        for act in (-1, 4, 100):
            refused(act=act)
    if form == "gated":                                       # one of G and U alone
        refused(change=(4, 0, 0))
        refused(change=(5, 0, 0))


@pytest.mark.parametrize("form", FORMS)
def test_calls_without_results_do_nothing(form):
    f, args = arguments(form, sizes=(0, N, K))
    assert f(*args) == b.GEMM_OK
    f, args = arguments(form, sizes=(M, 0, K))
    assert f(*args) == b.GEMM_OK


@pytest.mark.parametrize("form", FORMS)
def test_what_no_plan_takes_is_unsupported(form):
    big = (1 << 31) + 8
    f, args = arguments(form, sizes=(M, N, big))
    args = [big if 2 < j and a in (K,) else a for j, a in enumerate(args)]
    # Rows of K elements, or K rows: addresses far enough apart not to overlap.
    spread, seen = [], 0
    for a in args:
        if a in AT:
            seen += 1
            spread.append(seen << 44)
        else:
            spread.append(a)
    assert f(*spread) == UNSUPPORTED


def test_plans_and_their_hook():
    for op in range(5):
        for size in ((1, 14336, 4096), (16, 4096, 14336), (77, 130, 1), (2048, 11008, 4096), (5, 5, 0), (11008, 4096, 2048)):
            plan = ffn.ffn_plan(op, *size)
            k = -(-size[2] // 64) * 64 * (2 if op == ffn.FFN_OP_DX else 1)
            assert plan["config"] >= 0 and plan["name"].startswith("fused_") and plan["split_k"] >= 1
            assert plan["split_k"] * plan["k_chunk"] >= k and (k == 0 or (plan["split_k"] - 1) * plan["k_chunk"] < k)
        assert ffn.ffn_plan(op, 0, 5, 5)["config"] == -1
        for bad in ((-1, 1, 1), (1, -1, 1), (1, 1, -1)):
            with pytest.raises(b.GemmError):
                ffn.ffn_plan(op, *bad)
        with pytest.raises(b.GemmError) as e:
            ffn.ffn_plan(op, 1 << 31, 1, 1)
        assert e.value.status == UNSUPPORTED
        with pytest.raises(b.GemmError) as e:           # more workgroups than a launch holds
            ffn.ffn_plan(op, (1 << 31) - 5000, (1 << 31) - 5000, 1)
        assert e.value.status == UNSUPPORTED
        try:
            assert ffn.ffn_force_plan(op, 0, 3) == b.GEMM_OK
            plan = ffn.ffn_plan(op, 5, 5, 3000)
            assert plan["config"] == 0 and plan["split_k"] == 3
        finally:
            assert ffn.ffn_force_plan(op) == b.GEMM_OK
    for bad in ((5, -1, 0), (-1, -1, 0), (0, 64, 0), (0, -2, 0), (0, -1, -1)):
        assert ffn.ffn_force_plan(*bad) == BAD


def test_helpers_refuse_what_is_not_theirs():
    torch = pytest.importorskip("torch")
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="activations are"):
        b.gated_linear(x, w, w, "swish2")
    with pytest.raises(TypeError):
        b.gated_linear(x.float(), w, w)
    for call in (lambda: b.gated_linear(x, w, w), lambda: b.gated_linear_grad(x, w.t(), x, x), lambda: b.gated_linear_dx(x, w, x, w),
                 lambda: b.gated_linear_dw(x, x, x), lambda: b.linear_dw(x, x)):
        with pytest.raises(ValueError):                  # not on a GPU
            call()


@pytest.mark.parametrize("form", FORMS)
def test_negative_strides_past_64_bits_of_bytes_are_refused(form):
    """A stride whose bytes wrap round to a large positive number."""
    _, parts, _ = FORMS[form]
    for i, (_, _, size) in enumerate(p for p in parts if p != "act"):
        f, args = arguments(form, change=(i, None, -(1 << 64) // size + (1 << 30)))
        assert f(*args) == BAD, i
    good = [M, N, AT[0], N, AT[1], N, AT[2], N, 0, AT[3], N, AT[4], N]
    for i in (3, 5, 7, 10, 12):
        assert ffn.ffn_gated_bwd_bf16(*good[:i], -(1 << 63) + (1 << 30), *good[i + 1:]) == BAD, i
