"""Attention in blocks of 16 rows (GPU): a bf16 probability goes into the product
with the values in two parts.

Tolerances.  U = 2^-24, h = 2^-8 (bf16's half step).  With A = sum p |v| / sum p: a
score is off by at most (head_dim + 8) U of its terms' magnitudes, an exponential by
that much of itself and 8 U, each of the two sums over the keys by (keys + 16) U of
its magnitude.  Of a probability in [2^e, 2^(e+1)) the low part is below 2^(e-6) and
rounded once, by 2^(e-15) at most.  One rounding of the result: h of itself.  Where values cancel, A is many times the result, and a probability rounded
to bf16 once (h of A) would not pass."""
from __future__ import annotations

import math

import pytest

from tests.gpu_common import say
from tests.test_block_plan import attend as plan
from tests.test_block_plan import plans  # noqa: F401

torch = pytest.importorskip("torch")
U, H = 2.0 ** -24, 2.0 ** -8
CALLS = [(1, 1, 1), (1, 2, 4), (1, 7, 1), (1, 31, 8), (1, 90, 3), (1, 700, 4), (3, 60, 4), (5, 500, 3), (12, 20, 1), (1, 3000, 1)]   # n, past, group


@pytest.mark.parametrize("D", [64, 128])
def test_these_calls_take_blocks_of_16_rows(plans, D):  # noqa: F811
    got = {}
    for n, past, group in CALLS:
        rows, splits, _ = plan(plans, D, "bf16", 4, n, group, -(-(past + n) // 16) * 16)
        assert rows == 16, (n, past, group)
        got[splits > 1] = True
    assert len(got) == 2


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,past,group", CALLS)
def test_errors_are_those_of_the_results_rounding(D, n, past, group):
    from tests.test_gpu_paged import BF16, Cache, gen, ints
    g = gen(n + past)
    c = Cache(g, 2, 2, D, BF16, 16, -(-(past + n) // 16))
    c.fill([past + n] * 2)
    q = c.rand(n, 2 * group)
    say(f"attend bf16 {D}: {n} of group {group} over {past}")
    got = c.c.attend(q, ints(past, past)).double()
    at = torch.arange(past + n, device="cuda")
    see = at <= past + torch.arange(n, device="cuda")[:, None]
    for b in range(2):
        for hk in range(2):
            k, v, _ = c.held(b, at, hk)
            qq = q[b, :, hk * group:(hk + 1) * group].double().permute(1, 0, 2)
            p = torch.softmax((qq @ k.t() * D ** -0.5).masked_fill(~see, -math.inf), -1)
            big = (qq.abs() @ k.abs().t() * D ** -0.5).masked_fill(~see, 0).amax(-1, keepdim=True)
            want, A = p @ v, p @ v.abs()
            e = A * (2 * U * ((D + 8) * big + 16 + past + n) + 2.0 ** -15)
            off = (got[b, :, hk * group:(hk + 1) * group].permute(1, 0, 2) - want).abs() - (e + H * (want.abs() + e))
            assert bool((off <= 0).all()), f"{float(off.max())} past its tolerance"


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
def test_infinite_values_stay_infinities(D):
    """Of a key with the row's largest probability (1 as the kernel has it), and of keys with ever smaller ones."""
    from tests.test_gpu_paged import BF16, Cache, gen, ints
    for past, at in ((2, 0), (40, 33), (200, 77)):
        c = Cache(gen(past), 1, 1, D, BF16, 16, -(-(past + 1) // 16))
        for bits in (0, 1, 7, 8, 9, 60, 110, 120, 124):
            c.k.zero_()
            c.v.fill_(1.0)
            k, v = torch.zeros(1, 1, 1, D, device="cuda", dtype=BF16), torch.ones(1, 1, 1, D, device="cuda", dtype=BF16)
            k[..., 0] = -bits                           # a score of -bits log(2): a probability of 2^-bits
            v[..., 3], v[..., D - 1] = math.inf, -math.inf
            c.c.append(k, v, ints(at))
            q = torch.ones(1, 1, 1, D, device="cuda", dtype=BF16)
            got = c.c.attend(q, ints(past), scale=math.log(2.0))
            assert float(got[0, 0, 0, 3]) == math.inf and float(got[0, 0, 0, D - 1]) == -math.inf, bits
            rest = torch.ones(D, dtype=torch.bool, device="cuda")
            rest[[3, D - 1]] = False
            assert bool((got[0, 0, 0, rest] == 1).all()), bits
