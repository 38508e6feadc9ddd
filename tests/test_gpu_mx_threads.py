"""Two host threads with products on one stream: each call's copies of its operands, its K slices and its
product stay its own."""
import threading

import pytest
import torch

from paper_2512_13282_amd import binding as b
from paper_2512_13282_amd import mx
from test_gpu_mx import DEV, operands

pytestmark = pytest.mark.gpu


def work(op, M, N, K, seed):
    """A product over codes off 16-byte rows, which every call copies first."""
    a, codes, scales, cols = operands(op, M, N, K, seed)
    A = torch.from_numpy(a.view("int16")).to(DEV).view(torch.bfloat16)
    Q = mx.MxMatrix(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), cols)
    assert Q.codes.stride(0) % 16
    fn = {"fwd": b.linear_mx4, "dx": b.linear_mx4_dx, "dw": b.linear_mx8_dw}[op]
    return lambda: fn(A, Q, out_dtype=torch.float32)


@pytest.mark.parametrize("first,second", [(("fwd", 100, 515, 1027), ("fwd", 90, 515, 1027)),
                                          (("fwd", 70, 1001, 2049), ("dx", 33, 771, 900)),
                                          (("dw", 40, 515, 700), ("dx", 130, 515, 1000))])
def test_calls_of_two_threads_on_one_stream(first, second):
    calls = [work(*first, seed=1), work(*second, seed=2)]
    want = [c() for c in calls]
    torch.cuda.synchronize()
    wrong, start = [0, 0], threading.Barrier(2)

    def run(i):
        start.wait()
        for _ in range(10):
            for y in [calls[i]() for _ in range(20)]:
                wrong[i] += int(not torch.equal(y, want[i]))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert wrong == [0, 0]
