"""K slices of every block-scaled kernel in a captured call on a stream that holds no counters: a kernel of its
own adds the slices up, in the order in which the last slice of an eager call does, so the bits are
the same.  And the eager slices of tile kernels on several streams."""
import pytest
import torch

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import mx
from test_gpu_mx import DEV, OPS, configurations, operands

pytestmark = pytest.mark.gpu
FNS = {"fwd": b.linear_mx4, "dx": b.linear_mx4_dx, "dw": b.linear_mx8_dw}


def tensors(op, M, N, K, seed):
    a, codes, scales, cols = operands(op, M, N, K, seed)
    A = torch.from_numpy(a.view("int16")).to(DEV).view(torch.bfloat16)
    return A, mx.MxMatrix(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), cols)


def plans(op, M, N, K, split):
    """Each configuration that takes the rows, forced with `split` slices."""
    i = OPS.index(op)
    try:
        for config in configurations(op):
            assert mx.mx_force_plan(i, config, split) == b.GEMM_OK
            try:
                plan = mx.mx_plan(i, M, N, K)
            except b.GemmError:
                assert config < 2 and M > (16, 48)[config]
                continue
            assert plan["config"] == config and 1 < plan["split_k"] <= split
            yield plan
    finally:
        mx.mx_force_plan(i)


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("size,split", [((13, 130, 1537), 3), ((77, 390, 1100), 2), ((300, 270, 1537), 3)],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_captured_slices_give_the_eager_bits(op, size, split, dtype):
    M, N, K = size
    A, Q = tensors(op, M, N, K, sum(size))
    out = torch.empty(M, N + 3, dtype=dtype, device=DEV)[:, :N]
    s = torch.cuda.Stream()
    ran = 0
    for plan in plans(op, M, N, K, split):
        torch.cuda.synchronize()
        assert b.gemm_release_workspace() == b.GEMM_OK          # and with it every counter
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            FNS[op](A, Q, out=out)
        for i in range(3):
            A.normal_()
            want = FNS[op](A, Q, out_dtype=dtype)
            out.fill_(7.0)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), (plan, i)
        del graph
        ran += 1
    assert ran >= 6
    torch.cuda.synchronize()
    assert b.gemm_release_workspace() == b.GEMM_OK


@pytest.mark.parametrize("op", OPS)
@pytest.mark.parametrize("size,split", [((40, 512, 4096), 7), ((300, 512, 1024), 4)],
                         ids=lambda v: "x".join(map(str, v)) if isinstance(v, tuple) else str(v))
def test_slices_give_the_same_bits_on_every_run_and_stream(op, size, split):
    M, N, K = size
    A, Q = tensors(op, M, N, K, sum(size))
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()]
    for plan in plans(op, M, N, K, split):
        torch.cuda.synchronize()
        results = []
        for _ in range(3):
            for s in streams:                                    # at the same time, each in its own workspace
                with torch.cuda.stream(s):
                    results.append(FNS[op](A, Q, out_dtype=torch.float32))
        torch.cuda.synchronize()
        for r in results[1:]:
            assert torch.equal(r, results[0]), plan
