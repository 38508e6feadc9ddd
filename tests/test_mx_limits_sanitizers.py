"""The limits of the block-scaled plans (long rows, large grids, strides) under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only), as test_mx_sanitizers.py runs the C ABI's tests."""
import os
import subprocess
import sys

from test_sanitizers import CSRC, HERE, ROOT, SAN, _env


def test_limits_under_sanitizers(tmp_path):
    out = str(tmp_path / "libgemm_host_san.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", *SAN, "-I", os.path.join(ROOT, "include"),
                    *(os.path.join(CSRC, f) for f in ("gemm_api.cpp", "selector.cpp", "mx_api.cpp", "mx_plan.cpp")),
                    os.path.join(HERE, "sanitize_stub.cpp"), os.path.join(HERE, "mx_stub.cpp"), "-o", out],
                   check=True, capture_output=True, text=True)
    code = ("import ctypes, itertools, sys; sys.path.insert(0, '.')\n"
            "from paper_2512_13282_amd import binding as b, mx\n"
            "sizes = [0, 1, 31, 48, 49, 4096, 1 << 21, (1 << 21) + 1, 1 << 23, 1 << 28, (1 << 31) - 4097, (1 << 31) - 4096, 1 << 31,\n"
            "         1 << 54, (1 << 63) - 1]\n"
            "n = 0\n"
            "for op, M, N, K in itertools.product(range(3), sizes, sizes, sizes):\n"
            "    info = mx.PlanInfo()\n"
            "    rc = mx.lib()['mx_plan'](op, M, N, K, ctypes.byref(info))\n"
            "    assert rc in (b.GEMM_OK, b.GEMM_ERR_UNSUPPORTED), rc\n"
            "    n += 1\n"
            "calls = (mx.mx_gemm_bf16_mx4_f32_bt, mx.mx_gemm_bf16_mx4_bf16, mx.mx_gemm_bf16_mx8_f32_at)\n"
            "strides = [0, 1, 64, 1 << 22, (1 << 22) + 1, 1 << 55, 1 << 62, -1]\n"
            "for fn, la, lq, size in itertools.product(calls, strides, strides, sizes):\n"
            "    rc = fn(5, size, 64, 1 << 12, la, 1 << 40, lq, 1 << 42, size if size < 1 << 30 else 64, 1 << 44, size)\n"
            "    assert rc in (b.GEMM_OK, b.GEMM_ERR_HIP, b.GEMM_ERR_INVALID_VALUE, b.GEMM_ERR_UNSUPPORTED), rc\n"
            "    n += 1\n"
            "print('ran', n)\n")
    r = subprocess.run([sys.executable, "-c", code], env=_env({"GEMM_MI355X_LIBRARY": out}), capture_output=True, text=True,
                       timeout=600, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert r.stdout.startswith("ran ")
