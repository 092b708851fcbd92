"""Attention over the paged cache in blocks of 64 and 128 rows, split and not, both
types: what only some keys of a tile do (values and keys that are no numbers, holes,
scores of -infinity), in pages smaller than a load's rows, than a tile and larger;
results in the queries' places.  CPU: each call runs the block it names, and every
choice of the plan is run by a call of the GPU tests."""
from __future__ import annotations

import math
import random

import pytest

from tests.gpu_common import say
from tests.test_block_plan import attend as plan
from tests.test_block_plan import plans  # noqa: F401

torch = pytest.importorskip("torch")
NAN = float("nan")

# type, width, rows of a block, split, n, past, group, page size: two entries of two key heads
CALLS = [
    ("bf16", 64, 64, False, 90, 0, 3, 2), ("bf16", 64, 64, False, 33, 50, 8, 128), ("bf16", 64, 64, True, 150, 300, 2, 16),
    ("bf16", 64, 64, True, 33, 500, 8, 128), ("bf16", 64, 128, False, 2600, 100, 8, 32), ("bf16", 64, 128, True, 257, 3700, 8, 64),
    ("bf16", 64, 128, True, 700, 3700, 3, 4),
    ("bf16", 128, 64, False, 70, 0, 4, 2), ("bf16", 128, 64, False, 40, 50, 8, 128), ("bf16", 128, 64, True, 90, 1000, 1, 16),
    ("bf16", 128, 64, True, 33, 300, 8, 128), ("bf16", 128, 128, False, 700, 100, 8, 128), ("bf16", 128, 128, True, 700, 1700, 2, 16),
    ("bf16", 128, 128, True, 257, 1700, 8, 64),
    ("f32", 64, 64, False, 90, 0, 3, 2), ("f32", 64, 64, False, 33, 50, 8, 64), ("f32", 64, 64, True, 130, 100, 2, 16),
    ("f32", 64, 64, True, 257, 100, 1, 128),
    ("f32", 128, 64, False, 70, 0, 4, 1), ("f32", 128, 64, False, 40, 50, 8, 64), ("f32", 128, 64, True, 90, 100, 3, 16),
    ("f32", 128, 64, True, 33, 300, 8, 128),
]
IDS = [f"{c[0]}_{c[1]}_{c[4]}x{c[6]}_over_{c[5]}_pages_{c[7]}" for c in CALLS]
CALL = "dtype,D,rows,split,n,past,group,ps"


def limit(n, past, ps):
    return -(-(past + n) // ps) * ps


@pytest.mark.parametrize(CALL, CALLS, ids=IDS)
def test_the_calls_take_their_blocks(plans, dtype, D, rows, split, n, past, group, ps):  # noqa: F811
    r, s, _ = plan(plans, D, dtype, 4, n, group, limit(n, past, ps))
    assert (r, s > 1) == (rows, split)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_choice_of_the_plan_is_run(plans, dtype):  # noqa: F811
    from tests import test_gpu_paged as g

    def choice(D, regions, n, group, positions, window=0, sinks=0):
        r, s, _ = plan(plans, D, dtype, regions, n, group, positions, window, sinks)
        return D, r, s > 1
    run = {choice(c[1], 4, c[4], c[6], limit(c[4], c[5], c[7])) for c in CALLS if c[0] == dtype}
    run |= {choice(D, 4, n, group, limit(n, past, 16)) for D in (64, 128) for n, past, group in g.LONG}
    run |= {choice(D, 6, n, group, past + n) for D in (64, 128) for group in (1, 3, 4) for n, past in g.CASES + g.WIDE}
    rng = random.Random(0)

    def size(most):
        return int(math.exp(rng.uniform(0, math.log(most + 1))))
    for _ in range(30000):
        D, regions, n, group, positions, window = rng.choice((64, 128)), size(2000), size(8000), rng.randint(1, 16), size(200000), rng.choice((0, size(4000)))
        assert choice(D, regions, n, group, positions, window, 4) in run, (D, regions, n, group, positions, window)


def cache(dtype, D, n, past, ps):
    from tests.test_gpu_paged import BF16, F32, Cache, gen
    c = Cache(gen(n + past), 2, 2, D, BF16 if dtype == "bf16" else F32, ps, limit(n, past, ps) // ps, heads_first=bool(n % 2))
    c.fill([past + n, past + n])
    return c


@pytest.mark.gpu
@pytest.mark.parametrize(CALL, CALLS, ids=IDS)
def test_attention(dtype, D, rows, split, n, past, group, ps):
    from tests.test_gpu_paged import check, ints, lengths
    c = cache(dtype, D, n, past, ps)
    q, pos = c.rand(n, 2 * group), ints(past, past)
    say(f"attend {dtype} {D}: {n} of group {group} over {past}, pages of {ps}")
    want = check(c, q, pos)
    check(c, q, pos, lengths(n, n // 3))
    check(c, q, pos, causal=False, scale=-0.1)
    check(c, q, pos, window=max(1, past // 2), sinks=3)
    again = q.clone()
    assert torch.equal(c.c.attend(again, pos, out=again), want)


@pytest.mark.gpu
@pytest.mark.parametrize(CALL, CALLS, ids=IDS)
def test_special_values_reach_the_rows_that_see_them(dtype, D, rows, split, n, past, group, ps):
    from tests.test_gpu_paged import check, ints, lengths
    c = cache(dtype, D, n, past, ps)
    q, pos = c.rand(n, 2 * group), ints(past, past)
    say(f"special values {dtype} {D}: {n} of group {group} over {past}, pages of {ps}")
    for at in (past + n // 2, past + n - 1):   # seen by the later half, by the last token
        k, v = c.rand(1), c.rand(1)
        v[0, 0, 0, 3], v[0, 0, 0, D - 1], v[0, 0, 1, 9], v[1, 0, 0, 5], k[1, 0, 1, 2] = math.inf, -math.inf, NAN, -math.inf, NAN
        c.c.append(k, v, ints(at, at))
        got = check(c, q, pos)
        assert bool(got[:, :at - past].isfinite().all()) or at != past + n // 2
        assert not bool(got[0, at - past:].isfinite().all())
    check(c, q, pos, lengths(n // 2 + 1, n - 1))
    check(c, q, pos, window=3, sinks=7)
    check(c, q, pos, window=50, sinks=9, causal=False)
    check(c, q, pos, causal=False)
    # (a query with an infinity has no softmax, and reaches no other row)
    q[0, n // 4, 0, 0] = math.inf
    got = c.c.attend(q, pos, lens=lengths(n // 2, n // 2))
    assert bool(got[0, n // 4, 0].isnan().all()) and bool(got[0, n // 4, 1:].isfinite().all()) and bool(got[0, :n // 4].isfinite().all())


@pytest.mark.gpu
@pytest.mark.parametrize(CALL, CALLS, ids=IDS)
def test_holes_and_scores_of_minus_infinity(dtype, D, rows, split, n, past, group, ps):
    from tests.test_gpu_paged import check, ints
    c = cache(dtype, D, n, past, ps)
    q, pos = c.rand(n, 2 * group), ints(past, past)
    say(f"holes {dtype} {D}: {n} of group {group} over {past}, pages of {ps}")
    last = c.per - 1
    c.table[0, last // 2], c.table[1] = -1, c.k.shape[0]
    if last > 1:
        c.table[0, 0] = 1 << 30
    got = check(c, q, pos)
    assert bool((got[1] == 0).all())
    check(c, q, pos, causal=False, window=20, sinks=30)
    check(c, q, pos, window=past + n, sinks=1)
    c.table[1] = c.table[0]
    q[0] = 0
    q[0, :, :, 0] = -math.inf
    c.k[..., 0] = 1
    got = check(c, q, pos)
    assert bool(got[1].isfinite().all()) and not bool((got[0].isfinite() & (got[0] != 0)).any())
