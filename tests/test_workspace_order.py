"""Calls of two host threads on one stream (CPU only): the launches of a call that hand data on through
the stream's workspace are queued one after the other, with no launch of the other call between them."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2512_13282_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC, ROOT = build.CSRC, build.ROOT


@pytest.fixture(scope="module")
def cases(tmp_path_factory):
    if shutil.which(build.HIPCC) is None:
        pytest.skip("no hipcc")
    tmp = tmp_path_factory.mktemp("order")
    objs = []
    for src in (os.path.join(HERE, "workspace_order.cpp"), os.path.join(CSRC, "gemm_launch.hip"), os.path.join(CSRC, "mx_gemm.hip"),
                os.path.join(CSRC, "mx_plan.cpp")):
        objs.append(str(tmp / (os.path.basename(src) + ".o")))
        subprocess.run([build.HIPCC, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIE", "-I",
                        os.path.join(ROOT, "include"), "-c", src, "-o", objs[-1]], check=True, capture_output=True, text=True)
    exe = str(tmp / "order")
    # The device code that the runtime would be handed is not there, and neither is the runtime.
    subprocess.run(["g++", *objs, "-pthread", "-Wl,--unresolved-symbols=ignore-all", "-o", exe], check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    return dict(line.split(": ", 1) for line in r.stdout.splitlines())


# A copy of operands (c), a product (p), a separate reduction (r).
@pytest.mark.parametrize("name,launches", [("copied operand", "cp"), ("copied operand, slices", "cp"),
                                           ("dense, separate reduction", "pr"), ("captured slices", "pr")])
def test_a_calls_launches_stay_together(cases, name, launches):
    first, second = ([f"{t}{c}" for c in launches] for t in (1, 2))
    assert cases[name].split() in (first + second + ["ok"], second + first + ["ok"]), cases[name]


def test_calls_on_two_streams_do_not_wait_for_each_other(cases):
    # Each thread's first launch is out before the other's second.
    assert re.fullmatch(r"(1c 2c|2c 1c) (1p 2p|2p 1p) ok", cases["two streams"]), cases["two streams"]
