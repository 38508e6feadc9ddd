"""Resource use of the feed-forward and adapter kernels, as the built library's code object states it: their accumulators
and operands in flight stay in registers (no scratch), and a workgroup fits a compute unit as often as its launch
expects."""
from test_kernel_resources import LDS_LIMIT, kernels  # noqa: F401  (a fixture)


def _fused(kernels):  # noqa: F811
    return {n: k for n, k in kernels.items() if n.startswith("_ZN4gemm") and any(s in n for s in ("fused_", "adapters_", "gated_bwd"))}


def test_every_kernel_present(kernels):  # noqa: F811
    names = _fused(kernels)
    # Six operators; GATED and ADAPT have kernels for few rows too, at any address (four sizes, on and off dwords) and on
    # 16-byte rows (two).
    for stem, count in (("fused_tile_kernel", 12), ("fused_pingpong_kernel", 30), ("fused_decode_kernel", 16), ("fused_stream_kernel", 4),
                        ("adapters_shrink_kernel", 17), ("adapters_dw_kernel", 3), ("gated_bwd_kernel", 1), ("fused_realign_kernel", 1)):
        assert sum(stem in n for n in names) == count, stem


def test_nothing_spills(kernels):  # noqa: F811
    for n, k in _fused(kernels).items():
        assert int(k["private_segment_fixed_size"]) == 0 and int(k["vgpr_spill_count"]) == 0, n


def test_workgroups_fit_a_compute_unit(kernels):  # noqa: F811
    """Registers (512 a lane on each of four SIMDs, in blocks of eight) and LDS hold a workgroup; two of the 64 x 128 tiles',
    and two of the eight-wave kernels' for few rows of GATED."""
    for n, k in _fused(kernels).items():
        waves = int(k["max_flat_workgroup_size"]) // 64
        registers = -(-int(k["vgpr_count"]) // 8) * 8
        lds = int(k["group_segment_fixed_size"])
        assert lds <= LDS_LIMIT and -(-waves // 4) * registers <= 512, n
        if "fused_tile_kernelILi" in n and "ELi64ELi128E" in n:
            assert 2 * lds <= LDS_LIMIT and 2 * (waves // 4) * registers <= 512, n
