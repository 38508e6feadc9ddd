"""Rows longer than the tile kernels can step over (4 MiB of A or of codes): the plan is the decode kernel's
where that takes the rows, whatever a tile would cost."""
import pytest

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import mx

OPS = (mx.MX_OP_FORWARD, mx.MX_OP_INPUT_GRADIENT, mx.MX_OP_WEIGHT_GRADIENT)


def unsupported(*args):
    with pytest.raises(b.GemmError) as e:
        mx.mx_plan(*args)
    return e.value.status == b.GEMM_ERR_UNSUPPORTED


@pytest.mark.parametrize("M", [1, 2, 4, 8, 16, 17, 33, 48])
@pytest.mark.parametrize("N", [1, 16, 256, 4096, 14336])
def test_few_rows_of_any_length_run_on_the_decode_kernel(M, N):
    for K in ((1 << 21) + 1, 2200000, 110_000_000 // M):
        plan = mx.mx_plan(mx.MX_OP_FORWARD, M, N, K)
        assert plan["name"].startswith("mx_decode") and plan["bm"] >= M, plan
        assert plan["split_k"] * plan["k_chunk"] >= K and plan["k_chunk"] % 128 == 0


def test_every_row_count_takes_the_length_that_the_header_names():
    for M in range(1, 49):
        plan = mx.mx_plan(mx.MX_OP_FORWARD, M, 64, 110_000_000 // M)
        # A slice of A fits 64 KiB of LDS, each row with 16 bytes between it and the next.
        assert M * (2 * plan["k_chunk"] + 16) <= 65536


def test_more_rows_and_the_gradients_are_refused():
    assert unsupported(mx.MX_OP_FORWARD, 49, 64, 2200000)
    assert unsupported(mx.MX_OP_INPUT_GRADIENT, 1, 64, 2200000)             # rows of A
    assert unsupported(mx.MX_OP_INPUT_GRADIENT, 1, 9000000, 64)             # rows of codes
    assert unsupported(mx.MX_OP_WEIGHT_GRADIENT, 2200000, 64, 5)
    assert unsupported(mx.MX_OP_WEIGHT_GRADIENT, 64, 4200000, 5)
    for op in OPS:      # the longest rows that are taken
        for M, N, K in ((300, 64, 1 << 21), (300, 4 << 20, 64)):
            assert mx.mx_plan(op, *((N, M, K) if op == mx.MX_OP_WEIGHT_GRADIENT and N > 1 << 22 else (M, N, K)))["config"] >= 0


def test_a_forced_tile_is_refused_before_the_launch():
    tile = mx.mx_plan(mx.MX_OP_FORWARD, 300, 300, 4096)["config"]
    try:
        assert mx.mx_force_plan(mx.MX_OP_FORWARD, tile, 2) == b.GEMM_OK
        assert unsupported(mx.MX_OP_FORWARD, 4, 64, 2200000)
    finally:
        mx.mx_force_plan(mx.MX_OP_FORWARD)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(4, 5, 2200000), (16, 3, 2200001), (20, 4, 2100033)])
def test_products_over_long_rows(M, N, K):
    from test_gpu_mx import check_product
    check_product("fwd", M, N, K, False, seed=M)
    check_product("fwd", M, N, K, True, seed=M + 1, pads=(3, 0, 0, 0))
