"""The host code of the attention operators and of the flow decoder's options
under AddressSanitizer and UndefinedBehaviorSanitizer (CPU): carry4_runtime.hip
and flow_runtime.hip with the sanitizers on their host side only, the choice of
kernel within the driver itself, tests/asan_carry4.cpp."""
from __future__ import annotations

import os
import subprocess

import pytest

from tests.test_runtime_sanitized import CLANG, CSRC, HIPCC, ROOT, SAN_HOST, _run


def test_operators_and_options_under_sanitizers(tmp_path):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG)):
        pytest.skip("hipcc or ROCm's clang++ is not installed")
    if os.path.exists("/dev/kfd"):
        pytest.skip("the driver's pointers are not a device's: for machines without a GPU")
    from paper_2609_35115_amd import _build
    kernels = os.path.join(ROOT, "paper_2609_35115_amd", "_build", "libdc_so_flow_kernels.o")
    if not os.path.exists(kernels):
        _build.build()
    objs = []
    for src in ("carry4_runtime.hip", "flow_runtime.hip"):
        o = str(tmp_path / (os.path.splitext(src)[0] + ".o"))
        _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC",
              "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *SAN_HOST,
              "-I", os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, src), "-o", o])
        objs.append(o)
    drv, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    _run([CLANG, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(ROOT, "tests", "asan_carry4.cpp"), "-o", drv])
    _run([CLANG, "-fsanitize=address,undefined", "-o", exe, drv, *objs, kernels,
          "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=600)
    report = r.stdout + r.stderr
    assert r.returncode == 0, report[-4000:]
    assert "failures 0" in r.stdout, report[-4000:]
    assert "runtime error" not in report and "AddressSanitizer" not in report, report[-4000:]
