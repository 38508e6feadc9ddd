"""Products at the ends of what a launch and 32-bit indices hold: a plan whose grid is one, or
GEMM_ERR_UNSUPPORTED from the plan on."""
import re

import pytest
import torch

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import mx

OPS = (mx.MX_OP_FORWARD, mx.MX_OP_INPUT_GRADIENT, mx.MX_OP_WEIGHT_GRADIENT)


def threads(plan, M, N):
    """Threads along the grid's first dimension."""
    waves = re.search(r"_(\d+)x(\d+)x(\d+)$", plan["name"])
    per = 64 * (int(waves[1]) * int(waves[2]) * int(waves[3]) if waves else 8)
    tiles_n = -(-N // plan["bn"])
    if plan["name"].startswith("mx_decode"):
        return tiles_n * per
    return -(-M // plan["bm"]) * tiles_n * plan["split_k"] * per


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("M,N,K", [(1, 1 << 27, 32), (1, 1 << 28, 32), (48, 1 << 28, 32), (1, (1 << 31) - 4097, 32),
                                   (16, 1 << 30, 256), (1 << 28, 1, 32), ((1 << 31) - 4097, 1, 1), (1 << 19, 1 << 20, 64)])
def test_a_plans_grid_is_one_that_a_launch_takes(op, M, N, K):
    try:
        plan = mx.mx_plan(op, M, N, K)
    except b.GemmError as e:
        # Only where rows are too long for the operator, or the largest tiles too many.
        assert e.status == b.GEMM_ERR_UNSUPPORTED
        long_rows = max(2 * M if op == 2 else 2 * K, K // 2 if op == 0 else N // 2 if op == 1 else N) > 1 << 22
        assert long_rows or -(-M // 256) * -(-N // 256) * 512 >= 1 << 32
        return
    assert threads(plan, M, N) < 1 << 32, plan


def test_a_forced_grid_past_the_limit_is_refused():
    for config in (0, 2):
        assert mx.mx_force_plan(mx.MX_OP_FORWARD, config, 0) == b.GEMM_OK
        try:
            assert mx.mx_plan(mx.MX_OP_FORWARD, 1, 1 << 26, 32)["config"] == config
            with pytest.raises(b.GemmError) as e:
                mx.mx_plan(mx.MX_OP_FORWARD, 1, (1 << 27) if config == 0 else (1 << 29), 32)
            assert e.value.status == b.GEMM_ERR_UNSUPPORTED
        finally:
            mx.mx_force_plan(mx.MX_OP_FORWARD)


@pytest.mark.parametrize("op", OPS)
def test_sizes_end_where_the_header_says(op):
    for i in range(3):
        size = [8, 8, 8]
        size[i] = (1 << 31) - 4096
        with pytest.raises(b.GemmError) as e:
            mx.mx_plan(op, *size)
        assert e.value.status == b.GEMM_ERR_UNSUPPORTED


@pytest.mark.gpu
def test_a_weight_of_more_rows_than_the_decode_kernels_grid_holds():
    """2^27 + 40 rows of 32 codes: the last results are those of the last rows alone."""
    dev = torch.device("cuda:0")
    N, tail = (1 << 27) + 40, 300
    codes = torch.zeros(N, 16, dtype=torch.uint8, device=dev)
    gen = torch.Generator(device=dev)
    gen.manual_seed(1)
    codes[-tail:] = torch.randint(0, 256, (tail, 16), generator=gen, device=dev, dtype=torch.uint8)
    codes[:tail] = codes[-tail:]
    scales = torch.full((N, 1), 127, dtype=torch.uint8, device=dev)
    x = torch.randint(-4, 5, (1, 32), generator=gen, device=dev).to(torch.bfloat16)
    y = b.linear_mx4(x, mx.MxMatrix(codes, scales, 32), out_dtype=torch.float32)
    own = b.linear_mx4(x, mx.MxMatrix(codes[-tail:].clone(), scales[-tail:].clone(), 32), out_dtype=torch.float32)
    assert torch.equal(y[:, -tail:], own) and torch.equal(y[:, :tail], own)     # halves of integers: exact in any order
    assert not y[:, tail:-tail].any()
