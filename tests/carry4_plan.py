"""The attention operators' choice of kernel, compiled by itself for the host:
tests that mean to run one block shape say so and are held to it."""
import ctypes
import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """#include "carry4_plan.h"
extern "C" void plan(int D, int sinks, int ring, int64_t regions, int n, int group, int window, int bf16, int* out)
{
    const dcf::Plan4 p = dcf::plan4(D, sinks, ring, regions, n, group, window, bf16 != 0);
    out[0] = p.rows;
    out[1] = p.splits;
}
"""


@functools.lru_cache(None)
def _lib():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "plan.cpp"), os.path.join(d, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2609_35115_amd", "csrc"),
                        "-o", so, src], check=True)
        return ctypes.CDLL(so)


def plan(B, n, Hq, H, D, sinks, window, ring, dtype):
    """(rows of a block, key splits) of a call of n tokens of B entries."""
    out = (ctypes.c_int * 2)()
    _lib().plan(D, sinks, ring, ctypes.c_int64(B * H), n, Hq // H, window, int(dtype == "bf16"), out)
    return out[0], out[1]
