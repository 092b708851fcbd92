"""Which kernel the GPU tests' calls run (CPU): a change of the rules that takes
a test away from the block shape it is for fails here."""
from ctypes import byref

import pytest

from paper_2609_35115_amd import flow
from tests import test_gpu_carry4_edges as edges, test_gpu_carry4_wide as wide, test_gpu_flow_wide as flow_wide
from tests.carry4_plan import plan
from tests.test_carry4_args import carry


@pytest.mark.parametrize("shape,f32,bf16", edges.SHAPES)
def test_edge_shapes(shape, f32, bf16):
    B, n, Hq, H, D, sinks, w = shape
    assert plan(*shape, w + n, "f32") == f32 and plan(*shape, w + n, "bf16") == bf16


@pytest.mark.parametrize("B,n,Hq,H,D,sinks,window,ring", [
    (1, 1, 1, 1, 64, 0, 100_000, 100_000), (4, 1, 8, 2, 128, 4, 5000, 5000), (17, 40, 4, 4, 64, 3, 1800, 1840), (26, 100, 5, 5, 128, 0, 3100, 3200)])
def test_workspace_is_the_plans(B, n, Hq, H, D, sinks, window, ring):
    """Splits times (width + 2) floats a row, of the type that takes more."""
    c = carry(batch=B, heads=H, head_dim=D, sinks=sinks, ring=ring)
    s = max(plan(B, n, Hq, H, D, sinks, window, ring, dtype)[1] for dtype in ("f32", "bf16"))
    assert s > 1 and flow.flib().dc_carry4_workspace(byref(c), Hq, n, window) == s * B * n * Hq * (D + 2) * 4


def test_every_shape_is_reached():
    got = {(dtype, *((p[0], p[1] > 1))) for _, f, b in edges.SHAPES for dtype, p in (("f32", f), ("bf16", b))}
    assert got == {(d, r, s) for d in ("f32", "bf16") for r in (16, 64, 128) for s in (False, True)} - {("f32", 128, False), ("f32", 128, True)}


@pytest.mark.parametrize("call,f32,bf16", wide.BLOCKS)
def test_block_calls(call, f32, bf16):
    B, n, Hq, H, D, sinks, w, _, ring = call
    assert plan(B, n, Hq, H, D, sinks, w, ring, "f32") == f32 and plan(B, n, Hq, H, D, sinks, w, ring, "bf16") == bf16


@pytest.mark.parametrize("call,f32,bf16", wide.FAR)
def test_far_calls(call, f32, bf16):
    assert plan(*call, "f32") == f32 and plan(*call, "bf16") == bf16


@pytest.mark.parametrize("name", list(flow_wide.ARCHS))
def test_flow_calls(name):
    """Entries are streams times guidance branches; every call's carry has the same slots."""
    a, chunk, prompt = flow_wide.ARCHS[name]
    h, slots = a["heads"], (a["f_prompt"], a["f_retained"], a["f_retained"] + a["f_call"])
    for dtype in ("f32", "bf16"):
        assert plan(2 * flow_wide.B, a["f_call"], h, h, 64, *slots, dtype) == chunk
        assert plan(2, a["f_prompt"], h, h, 64, *slots, dtype) == prompt


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_splits_do_not_take_a_call_past_the_launch(D, dtype):
    """Few or many regions of few or many rows over up to 2^24 slots: no more than 2^20
    blocks by splitting (a launch has fewer than 2^24; from thousands of blocks a CU on
    splits balance nothing)."""
    split = 0
    for regions in (1, 7, 300, 5000, 300_000, 1 << 22, 1 << 24):
        for n in (1, 17, 56, 1000, 50_000, 1 << 26):
            for slots in (458, 100_000, 1 << 24):
                if regions * n > 1 << 28:
                    continue
                rows, splits = plan(regions, n, 1, 1, D, 0, slots, slots, dtype)
                blocks = regions * -(-n // rows)
                assert splits == 1 or blocks * splits <= 1 << 20, (regions, n, slots, blocks, splits)
                split += splits > 1
    assert split > 10
