"""Attention operators over a streaming carry held in 4 bits: what is measured.

Three operators that a serving program calls around the attention of a
streaming transformer (the flow decoder's DiT, a speech-token decoder in front
of it):

  norm_rope  RMS norms of queries and keys per head and the position rotation
             in one pass
  append     new keys and values into the carry: a turn's first tokens, which
             stay, and a ring of the tokens after them, 4-bit E2M1 elements
             with one power-of-two scale for 32 values; the values that the
             carry then holds come back through its read call
  attend     attention over the carry: the first tokens and a sliding window,
             causal per token or one window for a whole call (chunk calls)

`run` computes each in plain torch operations, or with `own` through the
package's entry points.  `exact` computes them in 64 bits.

Element format (OCP Microscaling: E2M1 elements, blocks of 32): a block's scale
is 2^e with the least integer e in [-126, 126] for which 6 * 2^e is at least
the block's largest magnitude; an element is the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e, ties to the even code.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    def nr(name, **k):
        return dict(dict(op="norm_rope", name=name, dtype="bf16", rot=k["D"], inter=False, packed=True, near=0, far=4096, ragged=False), **k)

    def ap(name, **k):
        return dict(dict(op="append", name=name, dtype="bf16", near=0, far=4096, ragged=False), **k)

    def at(name, **k):
        return dict(dict(op="attend", name=name, dtype="bf16", causal=True, near=k["sinks"] + k["window"], far=4096, ragged=False), **k)

    return [
        # one token for a few live streams: the launch is all there is
        nr("norm_rope_step_b4", B=4, n=1, Hq=8, Hk=8, D=64),
        # a flow-decoder call of 128 streams with both guidance branches, out of the fused projection's rows
        nr("norm_rope_call_b256", B=256, n=56, Hq=8, Hk=8, D=64),
        # full precision, ragged streams, half of each head rotated, in neighbouring pairs, positions of a day-long session
        nr("norm_rope_far_f32", B=3, n=1337, Hq=10, Hk=2, D=128, dtype="f32", rot=64, inter=True, packed=False, far=300_000_000, ragged=True),
        # a long prompt of a decoder with shared key heads
        nr("norm_rope_prompt", B=2, n=16384, Hq=32, Hk=8, D=128),
        # one token of 32 streams stored
        ap("append_step_b32", B=32, n=1, H=8, D=128, sinks=4, ring=4099),
        # a flow-decoder call of 128 streams with both branches: 302 prompt frames kept, a ring for two chunks and the call
        ap("append_call_b256", B=256, n=56, H=8, D=64, sinks=302, ring=160),
        # a long prompt stored
        ap("append_prompt", B=2, n=8192, H=8, D=128, sinks=64, ring=12352),
        # one token of one stream over a flow-sized carry: latency
        at("attend_step_b1", B=1, n=1, Hq=8, H=8, D=64, sinks=302, window=156),
        # one token of eight long sessions with shared key heads: reading the carry is the work
        at("attend_step_long", B=8, n=1, Hq=32, H=8, D=128, sinks=4, window=131000, far=2_000_000),
        # the flow decoder's chunk call, 128 streams with both branches
        at("attend_call_b256", B=256, n=56, Hq=8, H=8, D=64, sinks=302, window=100, causal=False),
        # a flush at a turn's end in full precision: a few streams, each with its own number of frames
        at("attend_flush_f32", B=3, n=13, Hq=12, H=4, D=64, sinks=57, window=211, dtype="f32", causal=False, ragged=True),
        # a long prompt, causal, with a window and first tokens
        at("attend_prompt", B=1, n=8192, Hq=16, H=4, D=128, sinks=64, window=4096),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    op = rng.choice(["norm_rope", "append", "attend", "attend"])
    D = rng.choice([64, 128])
    c = dict(op=op, D=D, dtype=rng.choice(["bf16", "bf16", "f32"]), near=rng.choice([0, 0, 7000]), far=log(64, 20_000_000), ragged=rng.random() < 0.4)
    H, group = log(1, 16), rng.choice([1, 1, 2, 3, 4, 8])
    B = log(1, 256)
    if op == "norm_rope":
        n = log(1, max(1, 600_000 // (B * H * (group + 1))))
        c.update(B=B, n=min(n, 16384), Hq=H * group, Hk=H, rot=rng.choice([D, D, D // 2, 16]), inter=rng.random() < 0.3,
                 packed=rng.random() < 0.5)
    elif op == "append":
        n = log(1, max(1, 120_000 // (B * H)))
        c.update(B=B, n=min(n, 8192), H=H, sinks=rng.choice([0, 1, log(1, 400)]))
        c["ring"] = c["n"] + log(1, 5000)
    else:
        step = rng.random() < 0.5
        n = 1 if step else log(2, 2000)
        keys = log(1, 100_000 if step else 5000)
        while B * H * keys * (n if n > 16 else 4) * group > 4e8 or B * n * H * group > 100_000 or B * H * (keys + n) > 6_000_000:
            B, n, keys = max(1, B // 2), max(1, n * 2 // 3), max(1, keys * 2 // 3)
            if B == 1 and n == 1:
                break
        c.update(B=B, n=n, Hq=H * group, H=H, sinks=rng.choice([0, 4, log(1, 400)]), window=keys, causal=rng.random() < 0.6)
    return c


# ------------------------------------------------------------------- inputs

def _rand(gen, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)


def _channels(gen, H, D):
    """Keys have a few channels larger than the others."""
    return torch.exp(0.5 * _rand(gen, H, D))


def _streams(case, gen):
    """(position of each stream's first token of the call, tokens of each stream).  The listed calls find
    their window full; a drawn one may find a turn that has only begun."""
    B, n = case["B"], case["n"]
    pos = case["near"] + torch.randint(0, case["far"] + 1, (B,), generator=gen, device="cuda", dtype=torch.int64)
    lens = torch.full((B,), n, device="cuda", dtype=torch.int32)
    if case["ragged"]:
        lens = torch.randint(0, n + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        lens[B // 2] = n
    return pos, lens


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, B, n, D = DT[case["dtype"]], case["B"], case["n"], case["D"]
    s = dict(case=case)
    s["pos"], s["lens"] = _streams(case, gen)
    if case["op"] == "norm_rope":
        Hq, Hk = case["Hq"], case["Hk"]
        x = (_rand(gen, B, n, Hq + 2 * Hk, D) * (0.5 + torch.rand(B, n, 1, 1, generator=gen, device="cuda"))).to(dt)
        s["q"], s["k"] = x[:, :, :Hq], x[:, :, Hq:Hq + Hk]
        if not case["packed"]:
            s["q"], s["k"] = s["q"].contiguous(), s["k"].contiguous()
        s["q_gain"], s["k_gain"] = 1 + 0.2 * _rand(gen, D), 1 + 0.2 * _rand(gen, D)
        r = case["rot"]
        s["freqs"] = (10000.0 ** (-torch.arange(r // 2, device="cuda", dtype=torch.float64) * 2 / r)).float()
        s["out"] = (torch.zeros(B, n, Hq, D, device="cuda", dtype=dt), torch.zeros(B, n, Hk, D, device="cuda", dtype=dt))
        return s
    H = case["H"]
    ch = _channels(gen, H, D)
    if case["op"] == "append":
        s["k"] = (_rand(gen, B, n, H, D) * ch).to(dt)
        s["v"] = _rand(gen, B, n, H, D).to(dt)
        return s
    # the tokens that a stream's carry holds: the first `sinks`, then `recent`
    # tokens from position `first` on, the call's own among them
    S, recent = case["sinks"], case["window"] + n
    total = s["pos"] + s["lens"]
    s["first"] = torch.maximum(torch.full_like(total, S), total - recent)
    s["held"] = (total - s["first"]).clamp(0, recent)
    s["kept"] = total.clamp(max=S)
    ch = ch[:, None]
    kv = [torch.empty(B, S + recent, H, D, device="cuda", dtype=dt) for _ in range(2)]
    for b in range(B) if B * recent > 100_000 else [slice(None)]:
        for i, x in enumerate(kv):
            y = torch.randn(x[b].shape, generator=gen, device="cuda", dtype=dt)
            x[b] = y * ch[:, 0].to(dt) if i == 0 else y
    s["k"], s["v"] = kv
    s["q"] = _rand(gen, B, n, case["Hq"], D).to(dt)
    s["out"] = torch.zeros(B, n, case["Hq"], D, device="cuda", dtype=dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm_rope":
        return s
    if own:
        from paper_2609_35115_amd.carry4 import Carry4
        ring = case["ring"] if case["op"] == "append" else case["window"] + case["n"]
        s["carry"] = Carry4(case["B"], case["H"], case["D"], sinks=case["sinks"], ring=ring)
    if case["op"] == "attend":   # the carry as earlier calls and this call's append have left it
        k, v, S = s.pop("k"), s.pop("v"), case["sinks"]
        if own:
            if S:
                s["carry"].append(k[:, :S], v[:, :S], torch.zeros_like(s["pos"]), lens=s["kept"].int())
            s["carry"].append(k[:, S:], v[:, S:], s["first"], lens=s["held"].int())
        else:
            s["kv4"] = [_encode(x.transpose(1, 2)) for x in (k, v)]
            i = torch.arange(S + case["window"] + case["n"], device="cuda")
            at = s["first"][:, None] + i - S
            s["held_at"] = torch.where(i < S, i.expand_as(at), at)
            s["valid"] = torch.where(i < S, i < s["kept"][:, None], i - S < s["held"][:, None])
    return s


# ------------------------------------------------------------- plain forms

def _quantise(x):
    """Block exponents and signed 4-bit codes (sign in bit 3) of x [..., D]."""
    y = x.float().unflatten(-1, (-1, 32))
    m, e = torch.frexp(y.abs().amax(-1, keepdim=True))
    e = torch.where(m <= 0.75, e - 3, e - 2).clamp(-126, 126)
    a = torch.ldexp(y.abs(), -e)
    code = (a > 0.25).to(torch.uint8)
    for border, ge in ((0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        code += (a >= border) if ge else (a > border)
    return e.squeeze(-1), (code + 8 * torch.signbit(y).to(torch.uint8)).flatten(-2)


def _encode(x):
    """x [B, H, T, D] as packed codes and scale bytes, a stream at a time."""
    codes = torch.empty(*x.shape[:-1], x.shape[-1] // 2, device=x.device, dtype=torch.uint8)
    scales = torch.empty(*x.shape[:-1], x.shape[-1] // 32, device=x.device, dtype=torch.uint8)
    for b in range(x.shape[0]) if x.numel() > 1 << 26 else [slice(None)]:
        e, c = _quantise(x[b])
        codes[b], scales[b] = c[..., ::2] + 16 * c[..., 1::2], (e + 127).to(torch.uint8)
    return codes, scales


def _decode(codes, scales):
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    grid = torch.cat([grid, -grid])
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    return torch.ldexp(grid[c].unflatten(-1, (-1, 32)), (scales.int() - 127)[..., None]).flatten(-2)


def _norm_rope(x, gain, pos, freqs, inter):
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * gain
    r = 2 * len(freqs)
    at = pos[:, None] + torch.arange(x.shape[1], device=x.device)
    angle = (at[..., None].double() * freqs.double())[:, :, None]
    c, s = angle.cos().float(), angle.sin().float()
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if inter else (y[..., :r // 2], y[..., r // 2:r])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., r:]], -1)


def _attend(s):
    case = s["case"]
    (B, n, Hq, D), H = s["q"].shape, case["H"]
    at = s["pos"][:, None] + torch.arange(n, device="cuda")
    key_at, S, w = s["held_at"][:, None], case["sinks"], case["window"]
    if case["causal"]:
        seen = (key_at <= at[..., None]) & ((key_at < S) | (key_at > at[..., None] - w))
    else:
        seen = (key_at < S) | (key_at >= s["pos"][:, None, None] - w)
    seen = seen & s["valid"][:, None]
    out = torch.empty(B, n, Hq, D, device="cuda", dtype=torch.float32)
    # a few streams at a time where all scores at once would not fit
    step = max(1, min(B, int(2e9 // (Hq * n * key_at.shape[-1]))))
    for b in range(0, B, step):
        i = slice(b, b + step)
        k, v = (_decode(c[i], e[i]) for c, e in s["kv4"])
        q = s["q"][i].float().transpose(1, 2).reshape(len(k), H, -1, D)   # [b, H, (group, n), D]
        score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * D ** -0.5
        score = score.unflatten(2, (Hq // H, n)).masked_fill_(~seen[i].expand(-1, n, -1)[:, None, None], -math.inf)
        score = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
        total = score.sum(-1, keepdim=True)
        o = torch.matmul(score.flatten(2, 3), v).unflatten(2, (Hq // H, n)) / total.clamp(min=1e-30)
        out[i] = o.flatten(1, 2).transpose(1, 2)
    return out


def run(s):
    case = s["case"]
    if own:
        lens = s["lens"] if case["ragged"] else None
        if case["op"] == "norm_rope":
            from paper_2609_35115_amd.carry4 import qk_norm_rope
            return qk_norm_rope(s["q"], s["k"], s["pos"], s["freqs"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=1e-6,
                                interleaved=case["inter"], lens=lens, out=s["out"])
        if case["op"] == "append":
            s["carry"].append(s["k"], s["v"], s["pos"], lens=lens)
            return s["carry"].read(s["pos"], case["n"], lens=lens, dtype=DT[case["dtype"]])
        return s["carry"].attend(s["q"], s["pos"], case["window"], lens=lens, causal=case["causal"], out=s["out"])
    here = (torch.arange(case["n"], device="cuda") < s["lens"][:, None])[:, :, None, None]
    dt = DT[case["dtype"]]
    if case["op"] == "norm_rope":
        return tuple(torch.where(here, _norm_rope(x, g, s["pos"], s["freqs"], case["inter"]).to(dt), o)
                     for x, g, o in ((s["q"], s["q_gain"], s["out"][0]), (s["k"], s["k_gain"], s["out"][1])))
    if case["op"] == "append":
        return tuple(torch.where(here, _decode(*_encode(x)), 0).to(dt) for x in (s["k"], s["v"]))
    return torch.where(here, _attend(s).to(dt), s["out"])


def work(case):
    """Of full streams: each input read once, each output written once."""
    B, n, D = case["B"], case["n"], case["D"]
    es = 2 if case["dtype"] == "bf16" else 4
    held = D // 2 + D // 32   # bytes of a key or value in the carry
    if case["op"] == "norm_rope":
        x = B * n * (case["Hq"] + case["Hk"]) * D
        return {"bytes": 2 * x * es, "flops": 8 * x}
    if case["op"] == "append":
        rows = 2 * B * n * case["H"]
        return {"bytes": rows * (2 * D * es + 2 * held), "flops": 4 * rows * D}
    w, S = case["window"], case["sinks"]
    if case["causal"]:
        keys, seen = S + w + n - 1, n * (S + w)
    else:
        keys, seen = S + w + n, n * (S + w + n)
    return {"bytes": 2 * B * n * case["Hq"] * D * es + 2 * B * case["H"] * keys * held, "flops": 4 * B * case["Hq"] * seen * D}


# ------------------------------------------------------------------- exact

def _exact_held(x):
    """The values that x [..., D] is held as, in 64 bits: round to the nearest
    multiple of the element's own step (half of its power of two, 0.5 at least)."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top / 6)).clamp(-126, 126)
    e = torch.where(6 * torch.exp2(e - 1) >= top, e - 1, e).clamp(min=-126)
    e = torch.where(6 * torch.exp2(e) < top, e + 1, e)
    y = y * torch.exp2(-e)
    step = torch.where(y.abs() >= 4, 2.0, torch.where(y.abs() >= 2, 1.0, 0.5))
    return (torch.round(y / step) * step * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    s = _inputs(case, seed)
    B, n, D = case["B"], case["n"], case["D"]
    lens = s["lens"].tolist()
    if case["op"] == "append":
        out = [_exact_held(s[x]) for x in ("k", "v")]
        for b in range(B):
            for o in out:
                o[b, lens[b]:] = 0
        return tuple(out)
    if case["op"] == "norm_rope":
        out = []
        for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
            x = x.double()
            x = x / (x.pow(2).sum(-1, keepdim=True) / D + 1e-6).sqrt() * gain.double()
            h = case["rot"] // 2
            z = torch.complex(x[..., 0:2 * h:2], x[..., 1:2 * h:2]) if case["inter"] else torch.complex(x[..., :h], x[..., h:2 * h])
            t = (s["pos"][:, None] + torch.arange(n, device="cuda")).double()[..., None, None] * s["freqs"].double()
            z = z * torch.polar(torch.ones_like(t), t)
            if case["inter"]:
                x[..., 0:2 * h:2], x[..., 1:2 * h:2] = z.real, z.imag
            else:
                x[..., :h], x[..., h:2 * h] = z.real, z.imag
            for b in range(B):
                x[b, lens[b]:] = 0
            out.append(x)
        return tuple(out)
    # attention, one stream and key head after the other, over the positions in order
    S, w, H, g = case["sinks"], case["window"], case["H"], case["Hq"] // case["H"]
    pos, first, held, kept = (s[x].tolist() for x in ("pos", "first", "held", "kept"))
    out = torch.zeros(B, n, case["Hq"], D, device="cuda", dtype=torch.float64)
    for b in range(B):
        m = lens[b]
        if m == 0:
            continue
        key_at = torch.cat([torch.arange(kept[b]), first[b] + torch.arange(held[b])]).cuda()
        at = (pos[b] + torch.arange(m)).cuda()[:, None]
        old = (at - w + 1) if case["causal"] else torch.full_like(at, pos[b] - w)
        bar = torch.zeros(m, len(key_at), device="cuda", dtype=torch.float64)
        bar[(key_at >= S) & (key_at < old)] = -math.inf
        if case["causal"]:
            bar[key_at > at] = -math.inf
        for h in range(H):
            k, v = (_exact_held(torch.cat([s[x][b, :kept[b], h], s[x][b, S:S + held[b], h]])) for x in ("k", "v"))
            q = s["q"][b, :m, h * g:(h + 1) * g].double().permute(1, 0, 2)
            p = torch.softmax(torch.matmul(q, k.t()) / math.sqrt(D) + bar, -1)
            out[b, :m, h * g:(h + 1) * g] = torch.matmul(p, v).permute(1, 0, 2)
    return out
