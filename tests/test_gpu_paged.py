"""The paged cache and its attention (GPU) against 64-bit references.

Tolerances.  U = 2^-24 is fp32's half step, h = finfo(type).eps / 2 a result's.
With A = sum p |v| / sum p: a score is off by at most (head_dim + 8) U of its
terms' magnitudes, an exponential by that much of itself and a few U, and each
of the two sums over the keys by (keys + 16) U of its magnitude.  In bf16 a
probability is rounded once more (h of itself) before both sums.  Results:
h of themselves."""
from __future__ import annotations

import math

import pytest

from tests.gpu_common import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Cache:
    """A PagedCarry with its pages in random order, unwritten rows NaN."""

    def __init__(self, g, B, H, D, dtype, ps, per, heads_first=False, extra=3):
        from paper_2609_35115_amd.paged import PagedCarry
        pages = B * per + extra
        self.table = torch.randperm(pages, generator=g, device="cuda")[:B * per].view(B, per).int()
        shape = (pages, H, ps, D) if heads_first else (pages, ps, H, D)
        self.k, self.v = (torch.full(shape, NAN, device="cuda", dtype=dtype) for _ in range(2))
        if heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        self.g, self.B, self.H, self.D, self.dtype, self.ps, self.per = g, B, H, D, dtype, ps, per
        self.c = PagedCarry(self.k, self.v, self.table)

    def rand(self, n, heads=None):
        return torch.randn(self.B, n, heads or self.H, self.D, generator=self.g, device="cuda").to(self.dtype)

    def fill(self, totals):
        """Stores random tokens [0, totals[b]) of every entry."""
        n = max(totals)
        if n:
            self.c.append(self.rand(n), self.rand(n), torch.zeros(self.B, device="cuda", dtype=torch.int64),
                          lens=torch.tensor(totals, device="cuda", dtype=torch.int32))

    def held(self, b, at, h):
        page = self.table[b].long()[at // self.ps]
        ok = (page >= 0) & (page < self.k.shape[0])
        page = page.clamp(0, self.k.shape[0] - 1)
        return self.k[page, at % self.ps, h].double(), self.v[page, at % self.ps, h].double(), ok


def reference(c, q, pos, lens, window, sinks, causal, scale):
    """(result, tolerance) in 64 bits, for rows within lens."""
    B, n, Hq, D = q.shape
    out = torch.zeros(B, n, Hq, D, device="cuda", dtype=torch.float64)
    tol = torch.zeros_like(out)
    group = Hq // c.H
    h = torch.finfo(c.dtype).eps / 2
    for b in range(B):
        m = n if lens is None else int(lens[b])
        p0 = int(pos[b])
        total = min(p0 + m, c.ps * c.per)
        if m == 0 or p0 < 0:
            continue
        at = torch.arange(max(total, 0), device="cuda")
        mine = p0 + torch.arange(m, device="cuda")[:, None]
        see = (at <= mine) if causal else torch.ones(m, len(at), dtype=torch.bool, device="cuda")
        if window:
            see = see & ((at < sinks) | (at > mine - window if causal else at >= p0 - window))
        for hk in range(c.H):
            k, v, ok = c.held(b, at, hk)
            s_ok = see & ok
            qq = q[b, :m, hk * group:(hk + 1) * group].double().permute(1, 0, 2)
            score = (qq @ k.t()) * scale
            size = ((qq.abs() @ k.abs().t()) * abs(scale)).masked_fill(~s_ok, 0)
            score = score.masked_fill(~s_ok, -math.inf)
            any_key = s_ok.any(-1)
            pr = torch.softmax(score, -1)
            pr = torch.where(s_ok, pr, 0.0)
            big = size.amax(-1, keepdim=True) if size.shape[-1] else torch.zeros(group, m, 1, device="cuda", dtype=torch.float64)
            # (0 times what a row does not see is 0)
            o = torch.zeros(group, m, D, device="cuda", dtype=torch.float64)
            A = torch.zeros_like(o)
            if len(at):
                fine = v.isfinite().all(-1)
                o = pr[..., fine] @ v[fine]
                A = pr[..., fine] @ v[fine].abs()
                for j in (~fine).nonzero().flatten().tolist():
                    o += torch.where(s_ok[:, j, None], pr[..., j, None] * v[j], 0.0)
            o[:, ~any_key] = 0
            e = A * (2 * U * ((D + 8) * big + 16 + len(at)) + (2 * h if c.dtype == BF16 else 0))
            out[b, :m, hk * group:(hk + 1) * group] = o.permute(1, 0, 2)
            tol[b, :m, hk * group:(hk + 1) * group] = (e + h * (o.abs() + e)).permute(1, 0, 2)
    return out, tol


def check(c, q, pos, lens=None, window=None, sinks=0, causal=True, scale=None, out=None):
    q0 = q.clone()
    got = c.c.attend(q, pos, window=window, lens=lens, sinks=sinks, causal=causal, scale=scale, out=out)
    want, tol = reference(c, q0, pos, lens, window, sinks, causal, c.D ** -0.5 if scale is None else scale)
    for b in range(c.B):
        m = q.shape[1] if lens is None else int(lens[b])
        x, w, t = got[b, :m].double(), want[b, :m], tol[b, :m]
        assert torch.equal(x.isnan(), w.isnan()), f"entry {b}: NaN in {int(x.isnan().sum())} places, not {int(w.isnan().sum())}"
        fine = w.isfinite()
        assert torch.equal(x[~fine & ~w.isnan()], w[~fine & ~w.isnan()]), f"entry {b}: infinities"
        off = ((x - w).abs() - t)[fine]
        assert bool((off <= 0).all()), f"entry {b}: {float(off.max())} past its tolerance"
    return got


def ints(*x):
    return torch.tensor(x, device="cuda", dtype=torch.int64)


def lengths(*x):
    return torch.tensor(x, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("ps,heads_first", [(1, False), (8, True), (64, False)])
def test_append_stores_what_is_there(dtype, ps, heads_first):
    g = gen(1)
    c = Cache(g, 3, 2, 64, dtype, ps, -(-40 // ps), heads_first)
    limit = c.ps * c.per
    c.table[1, 0] = -1                                  # holes
    c.table[2, c.per - 1] = c.k.shape[0]
    k, v = c.rand(11), c.rand(11)
    pos, lens = ints(0, 3, limit - 6), lengths(11, 7, 11)
    kept = c.k.clone(), c.v.clone()
    c.c.append(k, v, pos, lens=lens)
    for b in range(3):
        for i in range(int(lens[b])):
            x = int(pos[b]) + i
            page = int(c.table[b, x // ps]) if x < limit else -1
            if 0 <= page < c.k.shape[0]:
                kept[0][page, x % ps], kept[1][page, x % ps] = k[b, i], v[b, i]
    for a, b in zip(kept, (c.k, c.v)):
        assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))
    # positions that no caller may pass store nothing
    c.c.append(k, v, ints(-1, -5, 2 ** 62))
    for a, b in zip(kept, (c.k, c.v)):
        assert torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))


def test_append_takes_strided_rows():
    g = gen(2)
    for dtype in (BF16, F32):
        c = Cache(g, 2, 3, 64, dtype, 16, 4)
        fused = torch.randn(2, 20, 3 * 3 * 64 + 1, generator=g, device="cuda").to(dtype)[..., 1:].unflatten(-1, (9, 64))
        c.c.append(fused[:, :, 3:6], fused[:, :, 6:], ints(5, 30))
        for b, p in enumerate((5, 30)):
            for h in range(3):
                k, v, _ = c.held(b, torch.arange(p, p + 20, device="cuda"), h)
                assert torch.equal(k, fused[b, :, 3 + h].double()) and torch.equal(v, fused[b, :, 6 + h].double())


CASES = [(1, 1), (1, 40), (3, 1), (2, 7), (16, 33), (17, 5), (40, 100), (64, 64), (130, 65), (200, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 3])
def test_attend(dtype, D, group):
    """Calls of n tokens over `past` others, every mask, pages that end inside a tile."""
    g = gen(D + group)
    for n, past in CASES:
        say(f"attend {dtype} {D} group {group}: {n} over {past}")
        ps = 1 << int(torch.randint(0, 7, (), generator=g, device="cuda"))
        c = Cache(g, 3, 2, D, dtype, ps, -(-(past + n) // ps), heads_first=bool(n % 2))
        pos, lens = ints(past, past // 2, 0), lengths(n, n // 2, n)
        c.fill([past + n, past // 2 + n // 2, n])
        q = c.rand(n, 2 * group)
        check(c, q, pos, lens)
        check(c, q, pos, lens, causal=False)
        check(c, q, pos, lens, window=1)
        check(c, q, pos, lens, window=max(1, past // 2), sinks=past // 4, scale=0.2)
        check(c, q, pos, lens, window=5, sinks=2, causal=False)
        check(c, q, pos, lens, window=10_000, sinks=100, scale=-0.1)


LONG = [(1, 5000, 1), (1, 3001, 8), (4, 4100, 4), (5, 3000, 8), (70, 2600, 2), (600, 1500, 1), (40, 3000, 8), (24, 2500, 1), (1, 2000, 40), (2, 700, 23)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,past,group", LONG)
def test_attend_long_and_split(dtype, n, past, group):
    g = gen(n)
    for D in (64, 128):
        c = Cache(g, 2, 2, D, dtype, 16, -(-(past + n) // 16))
        c.fill([past + n, past // 3 + n])
        q = c.rand(n, 2 * group)
        say(f"attend {dtype} {D}: {n} of group {group} over {past}")
        check(c, q, ints(past, past // 3))
        check(c, q, ints(past, past // 3), window=1700, sinks=33, causal=False)
        check(c, q, ints(past, past // 3), window=300, sinks=33)


WIDE = [(700, 70), (2600, 100)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4])
def test_attend_wide(dtype, D, group):
    """Calls of many blocks of rows, in pages smaller and larger than a tile."""
    g = gen(D * group)
    for n, past in WIDE:
        for ps in (4, 128):
            c = Cache(g, 3, 2, D, dtype, ps, -(-(past + n) // ps), heads_first=ps == 4)
            lens = lengths(n, n - 1, n // 3)
            c.fill([past + n, past + n - 1, past + n // 3])
            q, pos = c.rand(n, 2 * group), ints(past, past, past)
            say(f"attend {dtype} {D} group {group}: {n} over {past}, pages of {ps}")
            check(c, q, pos, lens)
            check(c, q, pos, lens, window=200, sinks=9)
            check(c, q, pos, lens, window=50, sinks=100, causal=False)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 30, 150])
def test_rows_behind_and_in_place(dtype, n):
    g = gen(3)
    c = Cache(g, 4, 2, 64, dtype, 32, 10)
    pos, lens = ints(50, 9, 0, 120), lengths(n, 0, 1, n - 1)
    c.fill([50 + n, 9, 1, 120 + n - 1])
    q = c.rand(n, 4)
    want = check(c, q, pos, lens)
    q2 = q.clone()
    for b, m in enumerate(lens.tolist()):
        q2[b, m:] = NAN
    out = torch.full_like(q, 7.0)
    check(c, q2, pos, lens, out=out)
    check(c, q2, pos, lens, out=q2)
    for b, m in enumerate(lens.tolist()):
        assert torch.equal(out[b, :m], want[b, :m]) and torch.equal(q2[b, :m], want[b, :m])
        assert bool((out[b, m:] == 7.0).all()) and bool(q2[b, m:].isnan().all())
    # rows of a fused projection, not aligned to 16 bytes
    fused = torch.zeros(4, n, 4 * 64 + 1, device="cuda", dtype=dtype)[..., 1:].unflatten(-1, (4, 64))
    fused.copy_(q)
    check(c, fused, pos, lens, out=fused)
    for b, m in enumerate(lens.tolist()):
        assert torch.equal(fused[b, :m], want[b, :m])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 20, 100])
def test_special_values_reach_the_rows_that_see_them(dtype, n):
    """Infinities and NaN of later tokens, outside a window and in unwritten rows."""
    g = gen(n)
    for D in (64, 128):
        c = Cache(g, 2, 2, D, dtype, 16, 20)
        past = 60
        c.fill([past + n, past + n])
        k, v = c.rand(1), c.rand(1)
        v[0, 0, 0, 3], v[0, 0, 1, 9], v[1, 0, 0, 5], k[1, 0, 1, 2] = math.inf, NAN, -math.inf, NAN
        at = past + n // 2
        c.c.append(k, v, ints(at, at))                   # seen by the later half only
        q = c.rand(n, 4)
        got = check(c, q, ints(past, past))
        assert bool(got[:, :n // 2].isfinite().all()) and not bool(got[0, n // 2:].isfinite().all())
        check(c, q, ints(past, past), window=1)
        check(c, q, ints(past, past), window=3, sinks=7)
        check(c, q, ints(past, past), causal=False)
        # an infinite query has no softmax; it reaches no other row
        q[0, n - 1, 0, 0] = math.inf
        got = c.c.attend(q, ints(past, past), window=1)
        assert bool(got[0, n - 1, 0].isnan().all()) and bool(got[0, :n // 2].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,past", [(1, 100), (1, 3000), (90, 100), (90, 2000)])
def test_holes_and_rows_that_see_nothing(dtype, n, past):
    g = gen(past)
    c = Cache(g, 2, 1, 64, dtype, 16, -(-(past + n) // 16))
    c.fill([past + n] * 2)
    c.table[0, 1], c.table[0, 4] = -1, c.k.shape[0]
    c.table[1] = -7                                      # every key is a hole
    q = c.rand(n, 2)
    got = check(c, q, ints(past, past))
    assert bool((got[1] == 0).all())
    check(c, q, ints(past, past), window=200, sinks=20)
    # (entry 0's first page in a window's first tokens only)
    check(c, q, ints(past, past), window=2, sinks=40, causal=False)
    # every visible score is -infinity: no softmax (NaN), unlike a row that sees nothing
    c.table[1] = c.table[0].flip(0)
    c.table[1, 2] = -1
    q[0] = 0
    q[0, :, :, 0] = -math.inf
    c.k[..., 0] = 1
    got = check(c, q, ints(past, past))                  # (entry 1 sees rows of entry 0's last page that hold NaN)
    assert bool(got[0].isnan().all())
    c.table[1] = c.table[0]
    got = check(c, q, ints(past, past))
    assert bool(got[0].isnan().all()) and bool(got[1].isfinite().all())
    # positions past the table, and ones that no caller may pass
    limit = c.ps * c.per
    assert bool((c.c.attend(q, ints(limit + 5000, -3), window=100, out=torch.zeros_like(q)) == 0).all())


def test_prompt_pages_are_shared():
    """Two entries whose tables name the same prompt pages see the same keys."""
    g = gen(8)
    c = Cache(g, 2, 2, 128, BF16, 16, 6)
    c.table[1, :3] = c.table[0, :3]
    c.fill([48, 0])
    k, v = c.rand(5), c.rand(5)
    c.c.append(k, v, ints(48, 48))
    q = c.rand(5, 8)
    q[1] = q[0]
    k[1], v[1] = k[0], v[0]
    c.c.append(k, v, ints(48, 48))
    got = check(c, q, ints(48, 48))
    assert torch.equal(got[0], got[1])


def test_offsets_past_32_bits():
    """A pool whose last pages lie past 4 GiB and 2^31 elements."""
    from paper_2609_35115_amd.paged import PagedCarry
    g = gen(9)
    pages, ps, H, D = 9000, 64, 32, 128
    pool = torch.zeros(2, pages, ps, H, D, device="cuda", dtype=BF16)
    assert pool[0].numel() * 2 > 2 ** 32 and pool[0].numel() > 2 ** 31
    table = torch.tensor([[8999, 8998, 0]], device="cuda", dtype=torch.int32)
    c = PagedCarry(pool[0], pool[1], table)
    small = Cache(g, 1, H, D, BF16, ps, 3)
    for n, past in ((130, 0), (1, 130), (3, 131)):
        k, v, q = small.rand(n), small.rand(n), small.rand(n, 2 * H)
        for x in (c, small.c):
            x.append(k, v, ints(past))
        assert torch.equal(c.attend(q, ints(past)), check(small, q, ints(past)))


def test_captured_and_replayed():
    g = gen(10)
    c = Cache(g, 2, 2, 128, BF16, 64, 80)
    c.fill([5000, 4000])
    pos, lens = ints(4000, 3000), lengths(2, 2)
    k, v, q = c.rand(2), c.rand(2), c.rand(2, 8)
    out = torch.zeros_like(q)

    def calls():
        c.c.append(k, v, pos, lens=lens)
        c.c.attend(q, pos, lens=lens, out=out)           # keys split over blocks
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(3):
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        pos.add_(2)
        lens.copy_(lengths(2 - turn % 2, turn % 3))
        out.zero_()
        graph.replay()
        got = out.clone()
        out.zero_()
        calls()
        assert torch.equal(got, out), turn
        check(c, q, pos, lens)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_a_block_of_a_decoder(dtype):
    """The operators in a row, as a pre-norm block with a gated MLP runs them: two
    prompts in chunks and single tokens, against 64 bits."""
    from paper_2609_35115_amd.block import Norm, linear, norm_residual
    from paper_2609_35115_amd.carry4 import qk_norm_rope
    g = gen(13)
    B, W, Hq, H, D, M = 2, 256, 4, 2, 64, 320
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    qkv_w, o_w = (rnd((Hq + 2 * H) * D, W) * W ** -0.5).to(dtype), (rnd(W, Hq * D) * W ** -0.5).to(dtype)
    up_w, down_w, up_b = (rnd(2 * M, W) * W ** -0.5).to(dtype), (rnd(W, M) * M ** -0.5).to(dtype), 0.1 * rnd(2 * M)
    n1, n2, npost = Norm("rms", 1 + 0.1 * rnd(W)), Norm("rms", 1 + 0.1 * rnd(W)), Norm("rms", 1 + 0.1 * rnd(W))
    freqs = 10000.0 ** (-torch.arange(D // 2, device="cuda") * 2 / D)
    c = Cache(g, B, H, D, dtype, 16, 8)
    tokens = rnd(B, 40, W)
    outs = []
    for lo, hi in ((0, 17), (17, 38), (38, 39), (39, 40)):
        x, n, pos = tokens[:, lo:hi].contiguous(), hi - lo, ints(lo, lo)
        y = norm_residual(x, pre=n1, out=(None, torch.empty(B, n, W, device="cuda", dtype=dtype)))[1]
        qkv = linear(y, qkv_w).unflatten(-1, (Hq + 2 * H, D))
        q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        qk_norm_rope(q, k, pos, freqs, out=(q, k))
        c.c.append(k, v, pos)
        a = linear(c.c.attend(q, pos).flatten(2), o_w)
        x, y = norm_residual(x, a, post=npost, pre=n2)
        outs.append(linear(linear(y, up_w, up_b, act="silu_glu"), down_w, residual=x, out_dtype=F32))
    got = torch.cat(outs, 1).double()

    def rms(t, gain):
        t = t / (t.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        return t if gain is None else t * gain.double()
    x = tokens.double()
    qkv = (rms(x, n1.gain) @ qkv_w.double().t()).unflatten(-1, (Hq + 2 * H, D))
    ang = torch.arange(40, device="cuda").double()[:, None, None] * freqs.double()

    def rope(t):
        a, b = rms(t, None).chunk(2, -1)
        return torch.cat([a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()], -1)
    q, k, v = rope(qkv[:, :, :Hq]), rope(qkv[:, :, Hq:Hq + H]), qkv[:, :, Hq + H:]
    k, v = (t.repeat_interleave(Hq // H, 2).transpose(1, 2) for t in (k, v))
    s = q.transpose(1, 2) @ k.transpose(-1, -2) * D ** -0.5
    s = s.masked_fill(torch.ones(40, 40, device="cuda").triu(1).bool(), -math.inf)
    a = (torch.softmax(s, -1) @ v).transpose(1, 2).flatten(2) @ o_w.double().t()
    r = x + rms(a, npost.gain)
    u, w = (rms(r, n2.gain) @ up_w.double().t() + up_b.double()).chunk(2, -1)
    want = r + (u * torch.sigmoid(u) * w) @ down_w.double().t()
    rel = float((got - want).norm() / want.norm())
    # seven roundings to the type in a row, each at most h of values of the stream's own size, and an amplification of
    # a few by the norms; fp32 adds its sums' errors (256 terms)
    bound = 16 * 2.0 ** -8 if dtype == BF16 else 16 * 64 * U
    assert rel <= bound, (rel, bound)


def test_streams_and_threads():
    """Calls on two streams at once, each with its own workspace."""
    g = gen(14)
    cs = [Cache(g, 2, 2, 64, BF16, 32, 100) for _ in range(2)]
    qs = [c.rand(1, 8) for c in cs]
    for c in cs:
        c.fill([3000, 2500])
    want = [check(c, q, ints(2999, 2499)) for c, q in zip(cs, qs)]
    streams = [torch.cuda.Stream() for _ in cs]
    pos = ints(2999, 2499)
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, q, s in zip(cs, qs, streams):
            with torch.cuda.stream(s):
                got.append(c.c.attend(q, pos))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
