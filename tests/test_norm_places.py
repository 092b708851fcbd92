"""Norms whose results lie in their inputs' places (CPU): csrc/norm_plan.h's rule in a
model of a row that a block's waves load and store in any order, without a
barrier between them.  A row's last, partly filled vector is loaded as the row's
last eight elements, so that two threads have some of them."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """#include "norm_plan.h"
extern "C" int apart(const void* x, const void* h, const void* r, const void* y) { return dcb::results_apart(x, h, r, y); }
"""
ADDRESS = {"x": 1 << 20, "h": 2 << 20, "r": 3 << 20, "y": 4 << 20, None: 0}


@pytest.fixture(scope="module")
def apart(tmp_path_factory):
    d = tmp_path_factory.mktemp("norm")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2609_35115_amd", "csrc"),
                    "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    fn = ctypes.CDLL(str(d / "plan.so")).apart
    fn.argtypes = [ctypes.c_void_p] * 4
    return lambda **at: bool(fn(*(ADDRESS[at.get(k)] for k in ("x", "h", "r", "y"))))


def run(width, places, whole, backwards):
    """The results r = x + h and y = 3 r + 1 of a row: `places` says where each lies,
    `whole(result)` whether its repeated elements are stored.  Waves run one after
    the other, forwards or backwards."""
    vecs = (width + 7) // 8
    nv = 1 if vecs <= 256 else 2 if vecs <= 1024 else 4
    waves = -(-vecs // (64 * nv))
    memory = {"x": list(range(width)), "h": [7 * k % 11 for k in range(width)], "r": [None] * width, "y": [None] * width}
    for wave in range(waves)[::-1 if backwards else 1]:
        mine = [t + v * 64 * waves for t in range(64 * wave, 64 * wave + 64) for v in range(nv) if t + v * 64 * waves < vecs]
        firsts = {u: min(8 * u, width - 8) for u in mine}
        r = {u: [memory["x"][k] + memory["h"][k] if memory["h"] else memory["x"][k] for k in range(f, f + 8)] for u, f in firsts.items()}
        for result, value in (("r", lambda v: v), ("y", lambda v: 3 * v + 1)):
            if places.get(result) is None:
                continue
            to = memory[places[result]]
            for u, f in firsts.items():
                for j in range(0 if whole(result) else 8 * u - f, 8):
                    to[f + j] = value(r[u][j])
    return {result: memory[places[result]] for result in ("r", "y") if places.get(result)}


PLACES = [dict(r=r, y=y) for r in (None, "x", "h", "r") for y in (None, "x", "h", "y") if (r or y) and r != y]


@pytest.mark.parametrize("width", [1025, 1031, 1032, 1539, 2051, 2571, 4097, 16383])
@pytest.mark.parametrize("places", PLACES, ids=lambda p: f"r_{p['r']}_y_{p['y']}")
def test_results_in_any_place(apart, width, places):
    rule = apart(x="x", h="h", **places)
    assert rule == (not {"x", "h"} & set(places.values()))
    r = [k + 7 * k % 11 for k in range(width)]
    for backwards in (False, True):
        got = run(width, places, lambda _: rule, backwards)
        for name, want in (("r", r), ("y", [3 * v + 1 for v in r])):
            assert name not in got or got[name] == want, (name, backwards)


def test_without_h(apart):
    assert apart(x="x", y="y") and apart(x="x", r="r") and apart(x="x", r="r", y="y")
    assert not apart(x="x", r="x", y="y") and not apart(x="x", y="x")


def test_the_model_sees_a_rule_for_each_result_by_itself():
    """Which stores elements that another wave's result has taken the place of."""
    for places in (dict(r="x", y="y"), dict(r="h", y="y"), dict(r="r", y="x"), dict(r="r", y="h")):
        whole = {"r": places["r"] == "r", "y": places["y"] == "y"}.get
        r = [k + 7 * k % 11 for k in range(1025)]
        got = [run(1025, places, whole, backwards) for backwards in (False, True)]
        assert any(g["r"] != r or g["y"] != [3 * v + 1 for v in r] for g in got), places
