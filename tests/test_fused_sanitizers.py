"""The feed-forward and adapter C ABI and their plans under AddressSanitizer and UndefinedBehaviorSanitizer (CPU
only): a host-only build runs the CPU tests of the C ABI in a child process with the ASan runtime preloaded."""
import os
import subprocess
import sys

from test_sanitizers import CSRC, HERE, ROOT, SAN, _env

SOURCES = ("gemm_api.cpp", "selector.cpp", "mx_api.cpp", "mx_plan.cpp", "ffn_api.cpp", "adapters_api.cpp", "fused_plan.cpp")
STUBS = ("sanitize_stub.cpp", "mx_stub.cpp", "fused_stub.cpp")


def test_c_abi_under_sanitizers(tmp_path):
    out = str(tmp_path / "libgemm_host_san.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", *SAN, "-I", os.path.join(ROOT, "include"),
                    *(os.path.join(CSRC, f) for f in SOURCES), *(os.path.join(HERE, f) for f in STUBS), "-o", out],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-m", "not gpu", "-k", "not helpers",
                        os.path.join(HERE, "test_ffn_abi_cpu.py"), os.path.join(HERE, "test_adapters_abi_cpu.py")],
                       env=_env({"GEMM_MI355X_LIBRARY": out}), capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert " passed" in r.stdout
