"""Products over the whole range of scale bytes.  Every kernel has conversions of its own, so each
configuration runs: scales whose values are subnormal in bf16, the largest whose values are finite,
and those whose larger codes pass bf16's range and stand for infinities."""
import numpy as np
import pytest

import mx_reference as ref
from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import inputs, mx
from test_gpu_mx import OPS, configurations, run_product

pytestmark = pytest.mark.gpu

# 4-bit values reach 6 x 2^125 under byte 252, 8-bit ones 127 x 2^121 under byte 248.
LOW = (0, 1, 2, 3)
HIGH = {4: (249, 250, 251, 252), 8: (245, 246, 247, 248)}


def width(op):
    return 8 if op == "dw" else 4


def operands(op, M, N, K, seed, scale_bytes, a_power):
    """A's magnitudes lie around 2^a_power: products and sums are normal fp32 numbers."""
    rng = np.random.default_rng(seed)
    a = rng.standard_normal((K, M) if op == "dw" else (M, K))
    a = inputs.bf16_bits_from_f32((a * 2.0 ** a_power).astype(np.float32))
    rows, cols = (N, K) if op == "fwd" else (K, N)
    codes, scales = ref.random_packed(rows, cols, width(op), seed + 1)
    return a, codes, rng.choice(np.array(scale_bytes, np.uint8), size=scales.shape), cols


def over_configurations(op, M, N, K, splits=(1, 3)):
    ran = 0
    try:
        for config in configurations(op):
            for split in splits:
                assert mx.mx_force_plan(OPS.index(op), config, split) == b.GEMM_OK
                try:
                    plan = mx.mx_plan(OPS.index(op), M, N, K)
                except b.GemmError:
                    assert config < 2
                    continue
                ran += 1
                yield plan
    finally:
        mx.mx_force_plan(OPS.index(op))
    assert ran >= 6         # the operator with the fewest configurations has as many


SIZES = [(1, 40, 70), (13, 257, 331), (40, 130, 777), (150, 300, 515)]


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("end", ["low", "high"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_scales_at_both_ends(op, end, size):
    scale_bytes, power = (LOW, 60) if end == "low" else (HIGH[width(op)], -40)
    a, codes, scales, cols = operands(op, *size, sum(size), scale_bytes, power)
    want, magnitude = ref.product(op, ref.widen(a), ref.values(codes, scales, cols))
    lim = ref.bound(size[2], magnitude, want, False)
    for plan in over_configurations(op, *size):
        C = run_product(op, *size, a, codes, scales, False)
        off = np.abs(C - want)
        assert np.all(off <= lim), (plan, float((off / lim).max()), np.argwhere(~(off <= lim))[:4].tolist())
    C = run_product(op, *size, a, codes, scales, True)
    assert np.all(np.abs(C - want) <= ref.bound(size[2], magnitude, want, True))


@pytest.mark.parametrize("op", OPS)
def test_every_scale_byte(op):
    """Row by row (forward) or column block by column block, bytes 0 to the last that is finite for every
    code; A's rows hold one power of two each, which brings some of the results into fp32's range."""
    last = HIGH[width(op)][-1]
    blocks = last + 1
    if op == "fwd":
        M, N, K = 20, blocks, 32
    else:
        M, N, K = 20, 32 * blocks, 8
    rng = np.random.default_rng(7)
    codes, scales = ref.random_packed(*((N, K) if op == "fwd" else (K, N)), width(op), 8)
    scales[:] = np.arange(blocks)[:, None] if op == "fwd" else np.arange(blocks)[None, :]
    power = np.linspace(-120, 120, M).astype(int)
    av = rng.choice([-1.0, 1.0, 1.5], size=(M, K)) * np.exp2(power)[:, None]
    a = inputs.bf16_bits_from_f32((av if op != "dw" else av.T.copy()).astype(np.float32))
    want, magnitude = ref.product(op, ref.widen(a), ref.values(codes, scales, N if op != "fwd" else K))
    ok = (magnitude < 2.0 ** 127) & (magnitude > 2.0 ** -100)       # neither overflow nor subnormal sums
    assert ok.any(0).all()                                          # every byte is seen
    lim = ref.bound(K, magnitude, want, False)
    for plan in over_configurations(op, M, N, K, splits=(1,)):
        C = run_product(op, M, N, K, a, codes, scales, False)
        assert np.all((np.abs(C - want) <= lim)[ok]), plan


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("size", [(1, 33, 31), (5, 70, 95), (40, 130, 281), (150, 300, 517)], ids=lambda s: "x".join(map(str, s)))
def test_codes_past_the_end_are_no_part_of_the_sum(op, size):
    """Under bytes 253 and 254 the codes 4 and 6 are infinite.  The matrix holds none of them; what
    surrounds it (and the unused half of a row's last byte) does."""
    M, N, K = size
    a, codes, scales, cols = operands(op, M, N, K, sum(size), (253, 254) if op != "dw" else (249, 250), -60)
    if op == "dw":
        codes = (codes.astype(np.int64) % 32).astype(np.int8)
    else:
        codes = (codes & 0x99) | np.where(codes & 0x20, 0x22, 0).astype(np.uint8) & 0x22     # magnitudes 0, 1 (0.5), 2 (1), 3 (1.5)
        if cols % 2:
            codes[:, -1] = codes[:, -1] & 0x0f | 0x70
    want, magnitude = ref.product(op, ref.widen(a), ref.values(codes, scales, cols))
    assert np.all(np.isfinite(want))
    lim = ref.bound(K, magnitude, want, False)
    for plan in over_configurations(op, M, N, K):
        C = run_product(op, M, N, K, a, codes, scales, False)
        assert np.all(np.abs(C - want) <= lim), (plan, np.argwhere(~(np.abs(C - want) <= lim))[:4].tolist())


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("size", [(1, 96, 160), (20, 96, 200), (140, 260, 300)], ids=lambda s: "x".join(map(str, s)))
def test_values_past_the_range_are_infinite(op, size):
    """One value past bf16's range makes the results that use it infinite, of the product's sign, and no
    others."""
    M, N, K = size
    a, codes, scales, cols = operands(op, M, N, K, 5, (120, 121), 0)
    a = (a & 0x7fff) | 0x3f80                       # positive, none of them zero or not finite
    a = np.where((a & 0x7f80) >= 0x7f80, 0x3f80, a).astype(np.uint16)
    n, k = N // 3, K // 3
    r, c = (n, k) if op == "fwd" else (k, n)
    block = slice(c // 32 * 32, c // 32 * 32 + 32)
    scales = scales.copy()
    scales[r, c // 32] = 254
    if op == "dw":
        codes[r, block] = 0
        codes[r, c] = -127
    else:
        codes[r, c // 32 * 16:c // 32 * 16 + 16] = 0
        codes[r, c // 2] = 0xf << (4 * (c % 2))     # -6 x 2^127
    values = ref.values(codes, scales, cols)
    rest = values.copy()
    rest[r, c] = 0
    want, magnitude = ref.product(op, ref.widen(a), rest)
    lim = ref.bound(K, magnitude, want, False)
    others = np.arange(N) != n
    for plan in over_configurations(op, M, N, K, splits=(1,)):
        C = run_product(op, M, N, K, a, codes, scales, False)
        assert np.all(np.isneginf(C[:, n])), plan
        assert np.all((np.abs(C - want) <= lim)[:, others]), plan
