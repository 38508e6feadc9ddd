"""The feed-forward and adapter calls of two host threads on one stream, and a captured call whose stream's workspace
grows after the capture: each call hands sums, copies and h on through the workspace."""
import threading

import pytest
import torch

from paper_2512_13282_amd import adapters as ad
from paper_2512_13282_amd import binding as b
from test_gpu_ffn import BF16, DEV, generator, matrix

pytestmark = pytest.mark.gpu


def calls():
    gen = generator("threads")
    x, w = matrix(gen, 60, 1001), matrix(gen, 200, 1001)           # odd rows: copies
    A, B = matrix(gen, 3 * 8, 1001, 0.1).view(3, 8, 1001), matrix(gen, 3 * 200, 8, 0.1).view(3, 200, 8)
    index = torch.randint(-1, 3, (60,), generator=gen).to(torch.int32).to(DEV)
    v = matrix(gen, 1001, 200)
    return [lambda: b.gated_linear(x, w, w, "gelu"), lambda: b.linear_adapters(x, w, ad.Adapters(A, B), index, out_dtype=torch.float32),
            lambda: b.gated_linear_dx(x, v, x, v), lambda: b.linear_dw(x, x)]


def test_two_host_threads_on_one_stream():
    work = calls()
    want = [f() for f in work]
    torch.cuda.synchronize()
    stream, wrong = torch.cuda.Stream(), []

    def run(mine):
        with torch.cuda.stream(stream):
            got = [(i, work[i]()) for _ in range(40) for i in mine]
        stream.synchronize()
        wrong.extend(i for i, r in got if not torch.equal(r, want[i]))

    threads = [threading.Thread(target=run, args=(mine,)) for mine in ((0, 2), (1, 3))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_replays_after_the_workspace_has_grown():
    work = calls()
    want = [f() for f in work]
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for f in work:
            f()                                                    # the capture borrows the stream's counters
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        kept = [f() for f in work]
    big = torch.randn(700, 4001, device=DEV).to(BF16)
    with torch.cuda.stream(stream):
        grown = b.gated_linear(big, big, big)                      # larger copies than the workspace holds
    torch.cuda.synchronize()
    for _ in range(3):
        for k in kept:
            k.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in zip(kept, want):
            assert torch.equal(k, v)
        with torch.cuda.stream(stream):
            assert torch.equal(b.gated_linear(big, big, big), grown)
        torch.cuda.synchronize()
    del graph
