"""The matrix product's kernels, each split and not, with gated halves and without,
with rows of whole 16-byte chunks and of odd widths: every combination that the
plan chooses is run by a call (CPU: held to the plan; GPU: exact sums of whole
numbers, one rounding).  Calls planned for tiles that take whole chunks only, with
rows that do not begin at them, run the tile that takes any rows."""
from __future__ import annotations

import math
import random

import pytest

from tests.gpu_common import say
from tests.test_block_plan import FEW32, PLANE128, PLANE256, RING128, TILE128, TILE256
from tests.test_block_plan import linear as plan
from tests.test_block_plan import plans  # noqa: F401

torch = pytest.importorskip("torch")

# type, kernel, split, gated halves, batch, n, n_in, n_out
CALLS = [
    ("bf16", FEW32, True, 0, 2, 12, 2005, 41), ("bf16", FEW32, True, 0, 1, 20, 2048, 40), ("bf16", FEW32, True, 1, 1, 19, 1360, 31),
    ("bf16", FEW32, True, 1, 1, 19, 1302, 30),
    ("bf16", TILE128, True, 0, 1, 1699, 4936, 1212), ("bf16", TILE128, True, 0, 3, 399, 2987, 875), ("bf16", TILE128, True, 1, 2, 583, 5024, 851),
    ("bf16", TILE128, True, 1, 1, 193, 5705, 700), ("bf16", TILE128, True, 1, 2, 385, 2939, 630),
    ("bf16", TILE256, False, 0, 1, 1030, 176, 7209), ("bf16", TILE256, False, 1, 3, 429, 136, 2981), ("bf16", TILE256, False, 1, 1, 386, 144, 8511),
    ("bf16", TILE256, False, 1, 2, 1000, 1024, 4000), ("bf16", TILE256, True, 0, 1, 1475, 2576, 2752), ("bf16", TILE256, True, 0, 1, 129, 8192, 14336),
    ("bf16", TILE256, True, 1, 2, 737, 2608, 1375),
    ("bf16", RING128, False, 0, 2, 97, 40, 8239), ("bf16", RING128, False, 0, 1, 2048, 2048, 2048), ("bf16", RING128, False, 1, 1, 69, 24, 8326),
    ("bf16", RING128, True, 0, 11, 59, 3664, 477), ("bf16", RING128, True, 1, 1, 194, 3048, 690),
    ("f32", PLANE128, False, 0, 1, 199, 40, 12309), ("f32", PLANE128, True, 0, 2, 361, 1159, 643), ("f32", PLANE128, True, 1, 3, 107, 1047, 681),
    ("f32", PLANE256, False, 0, 4, 241, 293, 4116), ("f32", PLANE256, True, 0, 1, 534, 3232, 1028), ("f32", PLANE256, True, 0, 4, 322, 3043, 408),
    ("f32", PLANE256, True, 1, 1, 142, 2472, 1346), ("f32", PLANE256, True, 1, 1, 141, 2386, 1351), ("f32", PLANE256, True, 0, 1, 129, 2048, 8192),
]
IDS = [f"{c[0]}_{c[4]}x{c[5]}_{c[6]}_{c[7]}{'_glu' if c[3] else ''}" for c in CALLS]


@pytest.mark.parametrize("dtype,kind,split,glu,B,n,K,N", CALLS, ids=IDS)
def test_the_calls_run_their_kernels(plans, dtype, kind, split, glu, B, n, K, N):  # noqa: F811
    k, s, _ = plan(plans, B * n, K, N, dtype, glu)
    assert (k, s > 1) == (kind, split)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_choice_of_the_plan_is_run(plans, dtype):  # noqa: F811
    from tests import test_gpu_block as g
    calls = [(b * n, K, N, glu) for b, n in g.ROWS for K, N in g.SIZES for glu in (0, 1)] + [(b * n, K, N, glu) for b, n, K, N in g.TILES for glu in (0, 1)]
    calls += [(c[4] * c[5], c[6], c[7], c[3]) for c in CALLS if c[0] == dtype]

    def choice(M, K, N, glu):
        k, s, _ = plan(plans, M, K, N, dtype, glu)
        return k, s > 1, glu, K % 8 != 0
    run = {choice(*c) for c in calls}
    rng = random.Random(0)

    def size(most):
        return int(math.exp(rng.uniform(0, math.log(most + 1))))
    for _ in range(60000):
        M, K, N, glu = size(20000), size(16384), size(16384), rng.randint(0, 1)
        K = K if rng.random() < 0.4 else -(-K // 8) * 8
        assert choice(M, K, N, glu) in run, (M, K, N, glu)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind,split,glu,B,n,K,N", CALLS, ids=IDS)
def test_whole_numbers(dtype, kind, split, glu, B, n, K, N):
    from tests.test_gpu_block import BF16, F32, check_linear, gen, whole
    dt = BF16 if dtype == "bf16" else F32
    g = gen(K + N)
    say(f"linear {B} x {n}: {K} -> {N} {dtype} glu {glu} kernel {kind} split {split}")
    x = whole(g, B, n, K, dtype=dt)
    lens = torch.randint(0, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    if glu:
        w = whole(g, 2 * N, K, dtype=dt, most=1)
        check_linear(x, w, whole(g, 2 * N), act="none_glu", exact=True, out_dtype=F32)
        check_linear(x, w, act="none_glu", lens=lens, exact=True, out_dtype=F32)
    else:
        w = whole(g, N, K, dtype=dt)
        check_linear(x, w, whole(g, N), residual=whole(g, B, n, N), exact=True, out_dtype=F32)
        check_linear(x, w, gate=whole(g, B, N), residual=whole(g, B, n, N, dtype=dt), residual_scale=2.0, lens=lens, exact=True)


OFF = [c for c in CALLS if c[1] in (TILE256, RING128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,kind,split,glu,B,n,K,N", OFF, ids=[i for i, c in zip(IDS, CALLS) if c in OFF])
def test_rows_that_begin_between_chunks(dtype, kind, split, glu, B, n, K, N):
    """The rows, then the weight, inside wider rows that begin two bytes off."""
    from tests.test_gpu_block import BF16, F32, check_linear, gen, strided, whole
    g = gen(K)
    say(f"linear {B} x {n}: {K} -> {N} glu {glu} planned kernel {kind} split {split}, off")
    x, w = whole(g, B, n, K, dtype=BF16), whole(g, N * (1 + glu), K, dtype=BF16, most=1)
    act = "none_glu" if glu else "none"
    want = check_linear(x, w, act=act, exact=True, out_dtype=F32)
    got = check_linear(strided(x, 1, 8), w, act=act, exact=True, out_dtype=F32)
    assert torch.equal(got, want)
    got = check_linear(x, strided(w[None], 3, 6)[0], act=act, exact=True, out_dtype=F32)
    assert torch.equal(got, want)
