"""Infinities and NaN in fp32 products of any number of rows (GPU): what the sum of
the products gives, an infinity or NaN, in every kernel; exact elsewhere, and the
bits of what they do not reach as they are without them."""
from __future__ import annotations

import math

import pytest

from tests.gpu_common import say
from tests.test_block_plan import FEW16, FEW32, PLANE64, PLANE128, PLANE256
from tests.test_block_plan import linear as plan
from tests.test_block_plan import plans  # noqa: F401

torch = pytest.importorskip("torch")
INF, NAN = math.inf, math.nan

# kernel, split, gated halves, batch, n, n_in, n_out
CALLS = [
    (FEW16, False, 0, 1, 16, 70, 30), (FEW32, False, 0, 1, 17, 70, 30), (PLANE64, False, 0, 1, 33, 70, 30), (PLANE64, False, 0, 3, 100, 33, 129),
    (PLANE64, False, 1, 2, 40, 96, 50), (PLANE64, True, 0, 1, 33, 344, 40), (PLANE64, True, 1, 1, 70, 1024, 33), (PLANE128, False, 1, 1, 67, 168, 8232),
    (PLANE128, True, 0, 1, 395, 1352, 833), (PLANE128, True, 1, 1, 261, 903, 806), (PLANE256, False, 0, 1, 964, 293, 4116), (PLANE256, True, 0, 1, 534, 3232, 1028),
    (PLANE256, True, 1, 1, 141, 2386, 1351),
]
IDS = [f"{c[3]}x{c[4]}_{c[5]}_{c[6]}{'_glu' if c[2] else ''}" for c in CALLS]


@pytest.mark.parametrize("kind,split,glu,B,n,K,N", CALLS, ids=IDS)
def test_the_calls_run_their_kernels(plans, kind, split, glu, B, n, K, N):  # noqa: F811
    k, s, _ = plan(plans, B * n, K, N, "f32", glu)
    assert (k, s > 1) == (kind, split)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,split,glu,B,n,K,N", CALLS, ids=IDS)
def test_sums_with_infinities(kind, split, glu, B, n, K, N):
    from paper_2609_35115_amd.block import linear
    from tests.test_gpu_block import gen, whole
    g = gen(K)
    say(f"infinities {B} x {n}: {K} -> {N} glu {glu} kernel {kind} split {split}")
    R = N * (1 + glu)
    act = "none_glu" if glu else "none"
    for values in ("whole", "random"):
        x, w = (whole(g, B, n, K), whole(g, R, K, most=1 if glu else 3)) if values == "whole" else (
            torch.randn(B, n, K, generator=g, device="cuda"), torch.randn(R, K, generator=g, device="cuda"))
        without = linear(x, w, act=act)
        want = x.double() @ w.double().t()
        a, c = x.clone(), w.clone()
        last, b = n - 1, B - 1
        a[0, 0, K // 2], a[0, 1, 0], a[0, 1, K - 1], a[b, last, K - 1], a[b, last - 1, 1], a[0, 3, 2] = INF, INF, -INF, -INF, NAN, INF
        c[R - 1, K - 2], c[R // 2, 3], c[2, K // 3] = INF, -INF, NAN
        rows = [(0, 0), (0, 1), (b, last), (b, last - 1), (0, 3)]
        for at in rows:
            want[at] = (a[at].double() * c.double()).sum(-1)
        for col in (R - 1, R // 2, 2):
            want[..., col] = (a.double() * c[col].double()).sum(-1)
        if glu:
            want = want[..., :N] * want[..., N:]
        got = linear(a, c, act=act)
        special = ~want.isfinite()
        assert torch.equal(got.isnan(), want.isnan()), f"{values}: NaN in {int(got.isnan().sum())} places, not {int(want.isnan().sum())}"
        assert torch.equal(got[special & ~want.isnan()].double(), want[special & ~want.isnan()])
        assert int((special & ~want.isnan()).sum()) > 0 and int(special.sum()) < special.numel()
        assert torch.equal(got[~special], without[~special])
        if values == "whole":
            assert torch.equal(got[~special], want[~special].float())


@pytest.mark.gpu
def test_largest_values():
    """Sums near the largest magnitude, and past it."""
    from paper_2609_35115_amd.block import linear
    big = torch.finfo(torch.float32).max
    for n in (16, 40):
        x, w = torch.zeros(1, n, 64, device="cuda"), torch.zeros(8, 64, device="cuda")
        x[..., 0], w[0, 0], w[1, 0], w[2, 0], w[3, 0] = big, 1.0, 2.0, -2.0, 0.5
        x[..., 1] = big
        w[4, 1] = 0.25
        w[5, 0], w[5, 1] = 2.0, -INF
        y = linear(x, w)[0].nan_to_num(nan=7.0, posinf=INF, neginf=-INF)
        assert torch.equal(y, torch.tensor([big, INF, -INF, big / 2, big / 4, 7.0, 0, 0], device="cuda").expand(n, 8)), n
