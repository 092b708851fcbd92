"""The host code of a block's operators under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): block_runtime.hip with the sanitizers on its
host side only, the choices of kernel within the driver itself,
tests/asan_block.cpp; and the gfx950 code objects of their kernels."""
from __future__ import annotations

import os
import subprocess

import pytest

from tests import test_code_objects as objects
from tests.test_runtime_sanitized import CLANG, CSRC, HIPCC, ROOT, SAN_HOST, _run

KERNELS = ["norm_kernels", "linear_kernels", "paged_kernels"]


def test_operators_under_sanitizers(tmp_path):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG)):
        pytest.skip("hipcc or ROCm's clang++ is not installed")
    if os.path.exists("/dev/kfd"):
        pytest.skip("the driver's pointers are not a device's: for machines without a GPU")
    from paper_2609_35115_amd import _build
    kernels = [os.path.join(ROOT, "paper_2609_35115_amd", "_build", f"libdc_so_{k}.o") for k in KERNELS]
    if not all(os.path.exists(k) for k in kernels):
        _build.build()
    obj, drv, exe = (str(tmp_path / x) for x in ("runtime.o", "driver.o", "driver"))
    _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC",
          "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", *SAN_HOST,
          "-I", os.path.join(ROOT, "include"), "-c", os.path.join(CSRC, "block_runtime.hip"), "-o", obj])
    _run([CLANG, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
          "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-c", os.path.join(ROOT, "tests", "asan_block.cpp"), "-o", drv])
    _run([CLANG, "-fsanitize=address,undefined", "-o", exe, drv, obj, *kernels,
          "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=600)
    report = r.stdout + r.stderr
    assert r.returncode == 0, report[-4000:]
    assert "failures 0" in r.stdout, report[-4000:]
    assert "runtime error" not in report and "AddressSanitizer" not in report, report[-4000:]


@pytest.mark.parametrize("name", KERNELS)
def test_code_objects(name, tmp_path):
    """No scalar-memory write, no packed fp32 operation, and matrix instructions where products are."""
    obj = os.path.join(objects.OBJDIR, f"libdc_so_{name}.o")
    if not os.path.exists(obj):
        pytest.skip(f"{name} is not built (__graft_entry__.build())")
    if not all(os.path.exists(f"{objects.LLVM}/{t}") for t in ("llvm-objcopy", "clang-offload-bundler", "llvm-objdump")):
        pytest.skip("ROCm LLVM tools are not installed")
    dis = objects._disassemble(obj, tmp_path)
    assert dis is not None
    assert not sorted({m.group(0) for m in objects.SCALAR_WRITE.finditer(dis)})
    assert not sorted({m.group(0) for m in objects.PACKED_F32.finditer(dis)})
    assert ("v_mfma" in dis) == (name != "norm_kernels")
