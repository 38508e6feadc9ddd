"""Resource use of the block-scaled kernels, as the built library's code object states it: their
accumulators and operands in flight stay in registers (no scratch), and a workgroup fits a
compute unit as often as its launch expects."""
from test_kernel_resources import LDS_LIMIT, kernels  # noqa: F401  (a fixture)


def _mx(kernels):  # noqa: F811
    return {n: k for n, k in kernels.items() if n.startswith("_ZN4gemm") and "mx_" in n}


def test_every_block_scaled_kernel_present(kernels):  # noqa: F811
    names = _mx(kernels)
    for stem, count in (("mx_pack_kernel", 2), ("mx_unpack_kernel", 2), ("mx_realign_kernel", 1), ("mx_decode_kernel", 2),
                        ("mx_fwd_kernel", 9), ("mx_rows_kernel", 4), ("mx_grad_kernel", 10)):
        assert sum(stem in n for n in names) == count, stem


def test_nothing_spills(kernels):  # noqa: F811
    for n, k in _mx(kernels).items():
        assert int(k["private_segment_fixed_size"]) == 0 and int(k["vgpr_spill_count"]) == 0, n


def test_workgroups_fit_a_compute_unit(kernels):  # noqa: F811
    """Registers (512 a lane on each of four SIMDs, in blocks of eight) and LDS hold a workgroup; two of the
    rows kernels' with 16 rows or an 8-bit operand."""
    for n, k in _mx(kernels).items():
        waves = int(k["max_flat_workgroup_size"]) // 64
        registers = -(-int(k["vgpr_count"]) // 8) * 8
        lds = int(k["group_segment_fixed_size"])
        assert lds <= LDS_LIMIT and -(-waves // 4) * registers <= 512, n
        if "mx_rows_kernelILi1ELi1E" in n or "mx_rows_kernelILi2E" in n:
            assert 2 * lds <= LDS_LIMIT and 2 * (waves // 4) * registers <= 512, n
