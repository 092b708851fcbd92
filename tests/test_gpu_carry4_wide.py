"""What only some block shapes of the attention over the 4-bit carry do: a row's
base that moves from tile to tile, score scales of zero and below, rows that are
read and written element by element, results over their own queries, regions past
2^31 bytes.  The shapes (which a CPU test holds to their kernels) are those of the
edges, where every block shape has one, split and not."""
import math

import pytest
import torch

import tests.test_gpu_carry4 as base
from tests.test_gpu_carry4 import DT, carry4, dense, held, index, near, rand, same
from tests.test_gpu_carry4_edges import each_shape, each_type

pytestmark = pytest.mark.gpu

def bits(a, b):
    return bool(torch.equal(a, b))   # (not the tensors themselves: a failure would print them)


LEVELS = [0.0, 12.0, 24.0, 32.0, 48.0, 64.0, 96.0]   # held exactly


@each_type
@each_shape
@pytest.mark.parametrize("causal", [True, False], ids=["causal", "call"])
def test_scores_that_move_the_base(shape, causal, dtype):
    """Scores of whole powers of two that rise, fall and jump from tile to tile, by
    rows of different signs and sizes; a level's values are ones in dimensions of
    its own, so each result is a level's share.

    A score's log2 is off by its scale's two roundings and its product's, 3 halves of a
    last place of 96 at most, a ratio by two scores'; sums of K keys by 4 (K + 16)
    2^-24; in bf16 a share by a probability's, a sum's and a result's rounding."""
    B, n, Hq, H, D, _, w = shape
    m = carry4()
    keys = w + n
    c = m.Carry4(B, H, D, sinks=0, ring=keys)
    q = torch.zeros(B, n, Hq, D)
    q[..., 0] = torch.tensor([1.0, 0.5, -1.0, 0.25])[(torch.arange(n)[:, None] + 3 * torch.arange(Hq)) % 4]
    tol = math.expm1(2 * 96 * 3 * 2.0 ** -24) + 4 * (keys + 16) * 2.0 ** -24
    if dtype == "bf16":
        tol = (1 + tol) * (1 + 2.0 ** -8) ** 3 - 1
    c64 = float(torch.tensor(math.log(2.0), dtype=torch.float32)) / math.log(2.0)
    for order in ([0, 1, 2, 3, 4, 5, 6], [6, 5, 4, 3, 2, 1, 0], [3, 0, 5, 1, 6, 2, 4]):
        level = torch.tensor(order)[torch.arange(keys) // 64 % 7]
        k, v = torch.zeros(keys, H, D), torch.zeros(keys, H, D)
        k[..., 0] = torch.tensor(LEVELS)[level][:, None]
        for d in range(0, D, 16):
            v[torch.arange(keys), :, d + level] = 1.0
        put = [x[None].expand(B, keys, H, D).to(DT[dtype]).cuda() for x in (k, v)]
        c.append(*put, index([0] * B))
        got = c.attend(q.to(DT[dtype]).cuda(), index([w] * B), w, causal=causal, scale=math.log(2.0)).double().cpu()
        at = torch.arange(n)[:, None] + w
        see = torch.ones(n, keys, dtype=torch.bool) if not causal else (torch.arange(keys) <= at) & (torch.arange(keys) > at - w)
        count = see.double() @ torch.nn.functional.one_hot(level, 7).double()                # [n][7]
        s = q[0, :, :, 0].double()[..., None] * torch.tensor(LEVELS).double() * c64            # [n][Hq][7]
        top = s.masked_fill((count == 0)[:, None], -math.inf).amax(-1, keepdim=True)
        share = count[:, None] * 2.0 ** (s - top)
        share = share / share.sum(-1, keepdim=True)
        want = torch.zeros(n, Hq, D, dtype=torch.float64)
        for d in range(0, D, 16):
            want[..., d:d + 7] = share
        near(got, want.expand(B, n, Hq, D), tol, 0.0)


@each_type
@each_shape
@pytest.mark.parametrize("scale", [0.0, -0.2])
def test_scales_that_turn_scores_around(shape, scale, dtype):
    B, n, Hq, H, D, sinks, w = shape
    m = carry4()
    T = sinks + w + 9
    k, v, q = rand((B, T + n, H, D), dtype, 1), rand((B, T + n, H, D), dtype, 2), rand((B, n, Hq, D), dtype, 3)
    c = m.Carry4(B, H, D, sinks=sinks, ring=w + n)
    c.memory.fill_(255)
    c.append(k[:, :T], v[:, :T], index([0] * B))
    c.append(k[:, T:], v[:, T:], index([T] * B))
    for causal in (True, False):
        out = c.attend(q, index([T] * B), w, causal=causal, scale=scale)
        for b in {0, B - 1}:
            want, bound, top = dense((held(k[b]), held(v[b])), q[b], range(T, T + n), 0, w, causal, sinks, scale)
            rel = 2.0 ** -8 if dtype == "bf16" else 0.0
            near(out[b], want, rel, (bound + rel * top * (1 + rel)) * (1 + rel))


@each_type
@each_shape
def test_rows_element_by_element(shape, dtype):
    """Queries and results that start at odd elements, apart by odd numbers of them,
    and heads before tokens, and results over their queries: the same bits."""
    B, n, Hq, H, D, sinks, w = shape
    m = carry4()
    c = m.Carry4(B, H, D, sinks=sinks, ring=w + n)
    k = rand((B, w + n, H, D), dtype, 1)
    c.append(k, k.flip(1), index([0] * B))
    q, pos = rand((B, n, Hq, D), dtype, 3), index([w] * B)
    want = c.attend(q, pos, w)
    assert torch.isfinite(want).all()

    def odd():
        return torch.full((B * n * Hq * (D + 1) + 1,), 5.0, dtype=q.dtype, device="cuda")[1:].view(B, n, Hq, D + 1)
    x, o = odd(), odd()
    x[..., :D] = q
    assert bits(c.attend(x[..., :D], pos, w, out=o[..., :D]), want)
    assert (o[..., D] == 5.0).all()                                  # nothing behind the rows
    assert bits(c.attend(x[..., :D], pos, w), want)           # either side alone
    assert bits(c.attend(q, pos, w, out=o[..., :D].zero_()), want)
    t = torch.empty(B, Hq, n, D, dtype=q.dtype, device="cuda").transpose(1, 2).copy_(q)
    assert bits(c.attend(t, pos, w, out=torch.zeros_like(t)), want)
    assert c.attend(t, pos, w, out=t) is t and bits(t, want)
    assert c.attend(q, pos, w, out=q) is q and bits(q, want)


BLOCKS = [   # as of test_attend_block_shapes, and what the calls run
    ((30, 64, 2, 2, 64, 0, 960, False, 1024), (64, 4), (64, 4)),      # a block's rows exactly, keys in whole tiles
    ((300, 64, 1, 1, 128, 0, 192, False, 256), (64, 1), (64, 1)),
    ((300, 64, 1, 1, 64, 0, 192, False, 256), (64, 1), (64, 1)),
    ((300, 63, 1, 1, 64, 1, 191, True, 260), (64, 1), (64, 1)),
    ((100, 16, 24, 8, 64, 3, 90, True, 200), (64, 1), (64, 1)),       # 48 rows: shared heads straddle the waves
    ((19, 380, 7, 7, 64, 70, 350, False, 800), (64, 1), (128, 1)),
    ((60, 256, 4, 4, 128, 0, 100, True, 400), (64, 1), (128, 1)),     # whole blocks of 128
]


@each_type
@pytest.mark.parametrize("call", [s for s, _, _ in BLOCKS], ids=["x".join(map(str, s)) for s, _, _ in BLOCKS])
def test_blocks(call, dtype):
    base.test_attend_block_shapes(*call, dtype)


FAR = [((1, 200, 7, 1, 128, 0, 2800, 1 << 24), (64, 11), (64, 11)), ((1, 4000, 7, 1, 128, 0, 1000, 1 << 24), (64, 1), (128, 2))]


@each_type
@pytest.mark.parametrize("call", [s for s, _, _ in FAR], ids=["64", "128"])
def test_wide_blocks_past_32_bits(call, dtype):
    """The largest region, 2.3 GB: tokens in its last slots and its first."""
    B, n, Hq, H, D, _, w, slots = call
    m = carry4()
    c = m.Carry4(B, H, D, sinks=0, ring=slots)
    assert c.bytes > 1 << 31
    first = slots - (w + n) // 2
    k, v, q = rand((B, w + n, H, D), dtype, 1), rand((B, w + n, H, D), dtype, 2), rand((B, n, Hq, D), dtype, 3)
    at = index([first])
    c.append(k, v, at)
    a, b = c.read(at, w + n)
    kv = held(k[0]), held(v[0])
    assert same(a[0], kv[0]) and same(b[0], kv[1])
    picked = [0, 1, n // 3, n // 2, n - 2, n - 1]
    for causal in (True, False):
        out = c.attend(q, index([first + w]), w, causal=causal)
        want, bound, top = dense(kv, q[0, picked], [first + w + i for i in picked], first, w, causal, 0)
        rel = 2.0 ** -8 if dtype == "bf16" else 0.0
        near(out[0, picked], want, rel, (bound + rel * top * (1 + rel)) * (1 + rel))
