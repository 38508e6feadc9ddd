"""The block-scaled C ABI and its plans (csrc/mx_api.cpp, csrc/mx_plan.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): a host-only build runs the CPU tests of the C ABI in a
child process with the ASan runtime preloaded."""
import os
import subprocess
import sys

from test_sanitizers import CSRC, HERE, ROOT, SAN, _env


def test_c_abi_under_sanitizers(tmp_path):
    out = str(tmp_path / "libgemm_host_san.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", *SAN, "-I", os.path.join(ROOT, "include"),
                    *(os.path.join(CSRC, f) for f in ("gemm_api.cpp", "selector.cpp", "mx_api.cpp", "mx_plan.cpp")),
                    os.path.join(HERE, "sanitize_stub.cpp"), os.path.join(HERE, "mx_stub.cpp"), "-o", out],
                   check=True, capture_output=True, text=True)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-m", "not gpu", "-k", "not helpers",
                        os.path.join(HERE, "test_mx_abi_cpu.py")],
                       env=_env({"GEMM_MI355X_LIBRARY": out}), capture_output=True, text=True, timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert " passed" in r.stdout
