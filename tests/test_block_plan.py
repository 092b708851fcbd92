"""The choice of kernel and splits of the matrix product and the paged attention
(CPU): compiled by itself for the host, held to the workspaces that the library
asks for, and every kernel is reached by a call of the GPU tests."""
import ctypes
import os
import subprocess
from ctypes import byref

import pytest

from paper_2609_35115_amd import flow
from tests.test_block_args import layer, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """#include "linear_plan.h"
#include "paged_plan.h"
extern "C" void linear(int64_t M, int N, int K, int glu, int bf16, int64_t* out)
{
    const dcb::LinearPlan p = dcb::plan_linear(M, N, K, glu, bf16);
    out[0] = p.kind, out[1] = p.splits, out[2] = p.ws_bytes;
}
extern "C" void paged(int D, int bf16, int64_t regions, int n, int group, int limit, int window, int sinks, int64_t* out)
{
    const dcb::PagedPlan p = dcb::plan_paged(D, bf16, regions, n, group, limit, window, sinks);
    out[0] = p.rows, out[1] = p.splits, out[2] = p.ws_bytes;
}
"""
FEW16, FEW32, TILE64, TILE128, TILE256, PLANE64, PLANE128, PLANE256, RING128 = range(9)


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2609_35115_amd", "csrc"),
                    "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    return ctypes.CDLL(str(d / "plan.so"))


def linear(plans, M, K, N, dtype, glu=0):
    out = (ctypes.c_int64 * 3)()
    plans.linear(ctypes.c_int64(M), N, K, glu, int(dtype == "bf16"), out)
    return tuple(out)


def attend(plans, D, dtype, regions, n, group, limit, window=0, sinks=0):
    out = (ctypes.c_int64 * 3)()
    plans.paged(D, int(dtype == "bf16"), ctypes.c_int64(regions), n, group, limit, window, sinks, out)
    return tuple(out)


@pytest.mark.parametrize("M,K,N,dtype,kind,split", [
    (4, 512, 1536, "bf16", FEW16, False), (16, 8192, 1024, "bf16", FEW16, True), (32, 512, 512, "bf16", FEW32, False),
    (32, 4096, 8192, "bf16", TILE64, True), (300, 1024, 1024, "bf16", TILE64, False), (14336, 2048, 512, "bf16", TILE128, False),
    (14336, 512, 2048, "bf16", TILE256, False), (8192, 8192, 8192, "bf16", TILE256, False), (3000, 3001, 3000, "bf16", TILE128, False),
    (4, 512, 1536, "f32", FEW16, False), (24, 1024, 1024, "f32", FEW32, None), (300, 1024, 1024, "f32", PLANE64, None),
    (4011, 1001, 777, "f32", PLANE128, False), (14336, 512, 2048, "f32", PLANE256, False), (128, 4096, 8192, "f32", PLANE128, True)])
def test_linear_kernels(plans, M, K, N, dtype, kind, split):
    k, s, ws = linear(plans, M, K, N, dtype)
    assert k == kind and split in (None, s > 1) and (ws == 0) == (s == 1)


@pytest.mark.parametrize("D,dtype,regions,n,group,limit,rows,split", [
    (64, "bf16", 4, 1, 1, 300, 16, False), (128, "bf16", 15, 1, 1, 1467, 16, True), (128, "f32", 8, 1, 4, 8000, 16, True),
    (64, "bf16", 128, 20, 1, 820, 16, False), (128, "f32", 50, 33, 1, 1263, 64, True), (128, "bf16", 114, 39, 8, 7018, 128, None),
    (128, "bf16", 8, 4096, 4, 10112, 128, False), (64, "bf16", 16, 8192, 1, 8192, 128, False), (64, "f32", 24, 2000, 2, 4000, 64, None)])
def test_attention_kernels(plans, D, dtype, regions, n, group, limit, rows, split):
    r, s, ws = attend(plans, D, dtype, regions, n, group, limit)
    assert r == rows and split in (None, s > 1) and (ws == 0) == (s == 1)


def test_workspaces_are_the_plans(plans):
    """Splits times rows of partial sums, padded to eight columns, with glu twice."""
    for M, K, N, glu in ((4, 8192, 100, 0), (4, 8192, 100, 1), (70, 4096, 64, 0), (128, 4096, 8192, 1), (9, 64, 64, 0)):
        for dtype, code in (("bf16", 1), ("f32", 0)):
            k, s, ws = linear(plans, M, K, N, dtype, glu)
            want = 0 if s == 1 else s * M * ((N + 7) // 8 * 8) * (2 if glu else 1) * 4
            m = layer(n_in=K, n_out=N, stride=K, dtype=code, glu=glu)
            assert ws == want == flow.flib().dc_linear_workspace(byref(m), 1, M)
    for D, heads, q, n, pages in ((64, 2, 4, 1, 4096), (128, 1, 8, 3, 1000), (128, 4, 4, 40, 300), (64, 3, 3, 1, 2)):
        for dtype, code in (("bf16", 1), ("f32", 0)):
            c = paged(batch=3, heads=heads, head_dim=D, dtype=code, table_pages=pages)
            for window, sinks in ((0, 0), (3000, 60)):
                r, s, ws = attend(plans, D, dtype, 3 * heads, n, q // heads, 16 * pages, window, sinks)
                want = 0 if s == 1 else 3 * q * n * s * (D + 2) * 4
                assert ws == want == flow.flib().dc_paged_workspace(byref(c), q, n, window, sinks)


def test_every_linear_kernel_is_run_by_the_gpu_tests(plans):
    from tests import test_gpu_block as g
    for dtype, kinds in (("bf16", {FEW16, FEW32, TILE64, TILE128, TILE256, RING128}), ("f32", {FEW16, FEW32, PLANE64, PLANE128, PLANE256})):
        calls = [(b * n, K, N, glu) for b, n in g.ROWS for K, N in g.SIZES for glu in (0, 1)] + [(b * n, K, N, glu) for b, n, K, N in g.TILES for glu in (0, 1)]
        got = {(k, s > 1) for k, s, _ in (linear(plans, *c[:3], dtype, c[3]) for c in calls)}
        assert {k for k, _ in got} == kinds and {(k, True) for k in kinds if k not in (TILE256, PLANE256)} <= got | {(TILE128, True)}, got


def test_every_attention_kernel_is_run_by_the_gpu_tests(plans):
    from tests import test_gpu_paged as g
    for dtype in ("bf16", "f32"):
        got = set()
        for D in (64, 128):
            for n, past, group in g.LONG:
                r, s, _ = attend(plans, D, dtype, 4, n, group, -(-(past + n) // 16) * 16)
                got.add((D, r, s > 1))
            for group in (1, 3, 4):
                for n, past in g.CASES + g.WIDE:
                    r, s, _ = attend(plans, D, dtype, 6, n, group, past + n)
                    got.add((D, r, s > 1))
        want = {(D, r) for D in (64, 128) for r in ((16, 64, 128) if dtype == "bf16" else (16, 64))}
        assert {x[:2] for x in got} == want and {x[:2] for x in got if x[2]} >= {(D, r) for D in (64, 128) for r in (16, 64)}, got
