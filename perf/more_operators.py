"""Operators of a transformer block over streaming calls: what is measured.

Four operators that a serving program calls around the attention operators
(the flow decoder's DiT block, a speech-token decoder in front of it), over
calls of `B` entries of `n` tokens, each entry with its own number of tokens
where the call is ragged:

  norm    the norm after a block, its gate and the residual's scale, and the
          modulated norm before the next block:
            r = x_scale x + gate post(h),   y = pre(r) (1 + scale) + shift
          with the residual stream in fp32 or bf16
  linear  out = residual + gate act(x W^T + bias), act none, GELU (tanh form),
          SiLU, or the product of an activated half with the other half
  append  new keys and values into a paged cache, through a table of pages
  attend  attention of a chunk of new tokens over the paged cache: causal or
          one window for the whole call, with first tokens that stay visible

`run` computes each in plain torch operations, or with `own` through the
package's entry points.  `exact` computes them in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def listed():
    def no(name, **k):
        return dict(dict(op="norm", name=name, dtype="bf16", res="bf16", h=True, post="rms", gate="none", pre="rms", mod="none", xs=1.0, ragged=False), **k)

    def li(name, **k):
        return dict(dict(op="linear", name=name, dtype="bf16", act="none", glu=False, bias=True, gate="none", res="none", out="bf16", ragged=False), **k)

    def ap(name, **k):
        return dict(dict(op="append", name=name, dtype="bf16", heads_first=False, ragged=False), **k)

    def at(name, **k):
        return dict(dict(op="attend", name=name, dtype="bf16", causal=True, window=0, sinks=0, heads_first=False, ragged=False), **k)

    return [
        # one token of four live streams between two sublayers: the launch is all there is
        no("norm_step_b4", B=4, n=1, C=1024),
        # the flow decoder's call of 128 streams with both guidance branches, its residual stream in fp32: LayerNorm
        # with a solver step's gate, scale and shift
        no("norm_call_b256", B=256, n=56, C=512, res="f32", post="none", gate="shared", pre="layer", mod="shared"),
        # long prompts of different lengths at an odd width (rows not aligned to 16 bytes), a modulation for each entry
        no("norm_prompt_odd", B=5, n=6001, C=2571, gate="entry", mod="entry", xs=0.5, ragged=True),
        # one token of four live streams through a fused QKV projection
        li("linear_step_b4", B=4, n=1, K=512, N=1536),
        # the flow decoder's MLP-up of 128 streams with both branches
        li("linear_call_gelu", B=256, n=56, K=512, N=2048, act="gelu"),
        # full precision, odd sizes, ragged entries, into a gated residual stream
        li("linear_odd_f32", B=3, n=1337, K=1001, N=777, dtype="f32", out="f32", gate="entry", res="f32", ragged=True),
        # the gated MLP-up of a decoder over a long prompt
        li("linear_prompt_glu", B=1, n=8192, K=4096, N=8192, act="silu", glu=True, bias=False),
        # one token of 32 streams stored
        ap("append_step_b32", B=32, n=1, H=8, D=128, ps=64, past=700),
        # a long prompt stored
        ap("append_prompt", B=2, n=8192, H=8, D=128, ps=64, past=100),
        # the last frames of a turn in full precision: a few streams, each with its own number of frames, one window for
        # the call
        at("attend_flush_f32", B=3, n=13, Hq=12, H=4, D=64, dtype="f32", ps=16, past=900, window=211, sinks=57, causal=False, ragged=True),
        # one token of eight long sessions with shared key heads: reading the cache is the work
        at("attend_step_long", B=8, n=1, Hq=32, H=8, D=128, ps=64, past=65000),
        # a chunk of a long prompt over what is already stored
        at("attend_chunk", B=2, n=4096, Hq=16, H=4, D=128, ps=128, past=6000),
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    def size(lo, hi):
        x = log(lo, hi)
        return x if x < 64 or rng.random() < 0.3 else x // 64 * 64

    op = rng.choice(["norm", "linear", "append", "attend"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.4)
    mods = ["none", "shared", "entry", "token"]
    B = log(1, 256)
    if op == "norm":
        C = size(8, 8192)
        n = log(1, max(1, 40_000_000 // (B * C)))
        c.update(B=B, n=min(n, 16384), C=C, res=rng.choice(["f32", c["dtype"]]), h=rng.random() < 0.8, xs=rng.choice([1.0, 0.7]),
                 post=rng.choice(["none", "rms", "layer"]), gate=rng.choice(mods), pre=rng.choice(["rms", "layer"]), mod=rng.choice(mods))
        if c["h"] and rng.random() < 0.2:
            c.update(pre="none", mod="none")
        if not c["h"]:
            c.update(post="none", gate="none")
    elif op == "linear":
        K, N = size(8, 8192), size(8, 8192)
        n = log(1, max(1, min(40_000_000 // (B * max(K, N)), int(1.5e11) // (B * K * N))))
        c.update(B=B, n=min(n, 16384), K=K, N=N, act=rng.choice(["none", "gelu", "silu"]), bias=rng.random() < 0.6, gate=rng.choice(mods),
                 res=rng.choice(["none", "f32", c["dtype"]]), out=rng.choice(["f32", c["dtype"]]), glu=False)
        c["glu"] = c["act"] != "none" and rng.random() < 0.4
    else:
        D, H, ps = rng.choice([64, 128]), log(1, 16), 2 ** rng.randint(3, 8)
        c.update(D=D, H=H, ps=ps, heads_first=rng.random() < 0.3)
        if op == "append":
            n = log(1, max(1, 120_000 // (B * H)))
            c.update(B=B, n=min(n, 8192), past=log(1, max(1, 120_000 // (B * H))))
        else:
            group, step = rng.choice([1, 1, 2, 3, 4, 8]), rng.random() < 0.5
            n = 1 if step else log(2, 3000)
            past = log(1, 100_000 if step else 8000)
            while B * H * group * n * (past + n) > 1e9 or B * H * (past + n) * D * (1 if c["dtype"] == "bf16" else 2) > 500_000_000 or B * n * H * group > 150_000:
                B, n, past = max(1, B // 2), max(1, n * 2 // 3), max(1, past * 2 // 3)
            c.update(B=B, n=n, Hq=H * group, past=past, causal=rng.random() < 0.7, window=rng.choice([0, 0, log(1, 4000)]), sinks=0)
            if c["window"]:
                c["sinks"] = rng.choice([0, 4, log(1, 400)])
    return c


# ------------------------------------------------------------------- inputs

def _rand(gen, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)


def _mod(kind, gen, B, n, C, centre=0.0):
    """A gate, scale or shift: one for all, one an entry, or one a token (as [., ., C])."""
    if kind == "none":
        return None
    shape = {"shared": (1, 1, C), "entry": (B, 1, C), "token": (B, n, C)}[kind]
    return centre + 0.3 * _rand(gen, *shape)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B, n, dt = case["B"], case["n"], DT[case["dtype"]]
    s = dict(case=case, lens=torch.full((B,), n, device="cuda", dtype=torch.int32))
    if case["ragged"]:
        s["lens"] = torch.randint(0, n + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        s["lens"][B // 2] = n
    if case["op"] == "norm":
        C, res = case["C"], DT[case["res"]]
        # a residual stream has a mean of its own and a few large channels
        s["x"] = ((_rand(gen, B, n, C) + 0.5) * torch.exp(0.5 * _rand(gen, C))).to(res)
        s["h"] = (2 * _rand(gen, B, n, C)).to(dt) if case["h"] else None
        for which in ("post", "pre"):
            kind = case[which]
            s[which + "_gain"] = None if kind == "none" else 1 + 0.2 * _rand(gen, C)
            s[which + "_bias"] = 0.2 * _rand(gen, C) if kind == "layer" else None
        s["gate"] = _mod(case["gate"], gen, B, n, C, 0.5)
        s["scale"], s["shift"] = _mod(case["mod"], gen, B, n, C), _mod(case["mod"], gen, B, n, C)
        s["out"] = (torch.zeros(B, n, C, device="cuda", dtype=res) if case["h"] else None,
                    torch.zeros(B, n, C, device="cuda", dtype=dt) if case["pre"] != "none" else None)
    elif case["op"] == "linear":
        K, N = case["K"], case["N"]
        s["x"] = _rand(gen, B, n, K).to(dt)
        s["w"] = (_rand(gen, N * (2 if case["glu"] else 1), K) * K ** -0.5).to(dt)
        s["bias"] = 0.3 * _rand(gen, s["w"].shape[0]) if case["bias"] else None
        s["gate"] = _mod(case["gate"], gen, B, n, N, 0.5)
        s["res"] = None if case["res"] == "none" else _rand(gen, B, n, N).to(DT[case["res"]])
        s["out"] = torch.zeros(B, n, N, device="cuda", dtype=DT[case["out"]])
    else:
        H, D, ps, past = case["H"], case["D"], case["ps"], case["past"]
        per = -(-(past + n) // ps)
        pages = B * per + 3
        s["table"] = torch.randperm(pages, generator=gen, device="cuda")[:B * per].view(B, per).int()
        s["pos"] = torch.full((B,), past, device="cuda", dtype=torch.int64)
        if case["ragged"]:
            s["pos"] = torch.randint(0, past + 1, (B,), generator=gen, device="cuda", dtype=torch.int64)
        shape = (pages, H, ps, D) if case["heads_first"] else (pages, ps, H, D)
        s["pool"] = [_rand(gen, *shape, dtype=dt) for _ in range(2)]
        ch = torch.exp(0.5 * _rand(gen, H, 1, D)).to(dt)   # keys have a few channels larger than the others
        s["pool"][0] *= ch if case["heads_first"] else ch.transpose(0, 1)
        if case["heads_first"]:
            s["pool"] = [p.transpose(1, 2) for p in s["pool"]]
        if case["op"] == "append":
            s["k"], s["v"] = (_rand(gen, B, n, H, D).to(dt) for _ in range(2))
        else:
            s["q"] = _rand(gen, B, n, case["Hq"], D).to(dt)
            s["out"] = torch.zeros(B, n, case["Hq"], D, device="cuda", dtype=dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        if case["op"] == "norm":
            from paper_2609_35115_amd.block import Norm
            for which in ("post", "pre"):
                if case[which] != "none":
                    s[which] = Norm(case[which], s[which + "_gain"], s[which + "_bias"], eps=EPS)
        elif case["op"] in ("append", "attend"):
            from paper_2609_35115_amd.paged import PagedCarry
            s["carry"] = PagedCarry(*s["pool"], s["table"])
    return s


# ------------------------------------------------------------- plain forms

def _norm(x, kind, gain, bias):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
    return x if bias is None else x + bias


def _act(x, act):
    if act == "silu":
        return x * torch.sigmoid(x)
    if act == "gelu":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _plain_norm(s, here):
    case = s["case"]
    r = case["xs"] * s["x"].float()
    if case["h"]:
        h = _norm(s["h"].float(), case["post"], s["post_gain"], s["post_bias"])
        r = r + (h if s["gate"] is None else s["gate"] * h)
    y = None
    if case["pre"] != "none":
        y = _norm(r, case["pre"], s["pre_gain"], s["pre_bias"])
        if s["scale"] is not None:
            y = y * (1 + s["scale"]) + s["shift"]
    return tuple(None if o is None else torch.where(here, v.to(o.dtype), o) for v, o in zip((r, y), s["out"]))


def _plain_linear(s, here):
    case = s["case"]
    y = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["glu"]:
        a, b = y.chunk(2, -1)
        y = _act(a, case["act"]) * b
    else:
        y = _act(y, case["act"])
    if s["gate"] is not None:
        y = y * s["gate"]
    if s["res"] is not None:
        y = y + s["res"].float()
    return torch.where(here, y.to(s["out"].dtype), s["out"])


def _places(s, at):
    """(page, offset in it) of positions at [B, T]."""
    ps = s["case"]["ps"]
    return torch.gather(s["table"].long(), 1, at // ps), at % ps


def _plain_append(s, here):
    page, off = _places(s, s["pos"][:, None] + torch.arange(s["case"]["n"], device="cuda"))
    for pool, x in zip(s["pool"], (s["k"], s["v"])):
        if s["case"]["ragged"]:
            x = torch.where(here[..., None], x, pool[page, off])
        pool[page, off] = x
    return tuple(s["pool"])


def _plain_attend(s, here):
    case = s["case"]
    (B, n, Hq, D), H, S, w = s["q"].shape, case["H"], case["sinks"], case["window"]
    pos, total = s["pos"][:, None], (s["pos"] + s["lens"])[:, None]
    if w:   # the first tokens, then those that a query's window may hold
        first = (pos - w).clamp(min=S)
        at = torch.cat([torch.arange(S, device="cuda").expand(B, S), first + torch.arange(w + n, device="cuda")], 1)
    else:
        at = torch.arange(case["past"] + n, device="cuda").expand(B, -1)
    mine = (pos + torch.arange(n, device="cuda"))[..., None]
    seen = (at < total)[:, None].expand(-1, n, -1)
    if case["causal"]:
        seen = seen & (at[:, None] <= mine)
    if w:
        seen = seen & ((at[:, None] < S) | (at[:, None] >= (mine - w + 1 if case["causal"] else pos[..., None] - w)))
    page, off = _places(s, at.clamp(max=s["table"].shape[1] * case["ps"] - 1))
    k, v = (pool[page, off].float().transpose(1, 2) for pool in s["pool"])          # [B, H, T, D]
    q = s["q"].float().transpose(1, 2).reshape(B, H, -1, D)                         # [B, H, (group, n), D]
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(D ** -0.5).unflatten(2, (Hq // H, n))
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    o = torch.matmul(score.flatten(2, 3), v.contiguous()).unflatten(2, (Hq // H, n)) / score.sum(-1, keepdim=True).clamp(min=1e-30)
    return torch.where(here[..., None], o.flatten(1, 2).transpose(1, 2).to(s["out"].dtype), s["out"])


def run(s):
    case = s["case"]
    if own:
        lens = s["lens"] if case["ragged"] else None
        if case["op"] == "norm":
            from paper_2609_35115_amd.block import norm_residual
            return norm_residual(s["x"], s["h"], post=s.get("post"), gate=s["gate"], x_scale=case["xs"], pre=s.get("pre"),
                                 scale=s["scale"], shift=s["shift"], lens=lens, out=s["out"])
        if case["op"] == "linear":
            from paper_2609_35115_amd.block import linear
            return linear(s["x"], s["w"], s["bias"], act=case["act"] + ("_glu" if case["glu"] else ""), gate=s["gate"],
                          residual=s["res"], lens=lens, out=s["out"])
        if case["op"] == "append":
            s["carry"].append(s["k"], s["v"], s["pos"], lens=lens)
            return tuple(s["pool"])
        return s["carry"].attend(s["q"], s["pos"], window=case["window"] or None, lens=lens, sinks=case["sinks"],
                                 causal=case["causal"], out=s["out"])
    here = (torch.arange(case["n"], device="cuda") < s["lens"][:, None])[..., None]
    return {"norm": _plain_norm, "linear": _plain_linear, "append": _plain_append, "attend": _plain_attend}[case["op"]](s, here)


def work(case):
    """Of full entries: each input read once, each output written once."""
    B, n = case["B"], case["n"]
    es = {"bf16": 2, "f32": 4}
    t, e = B * n, es[case["dtype"]]
    rows = {"none": 0, "shared": 1, "entry": B, "token": t}
    if case["op"] == "norm":
        C, r = case["C"], es[case["res"]]
        b = t * C * (r + (e + r if case["h"] else 0) + (e if case["pre"] != "none" else 0))
        return {"bytes": b + 4 * C * (rows[case["gate"]] + 2 * rows[case["mod"]]), "flops": t * C * (8 * case["h"] + 8)}
    if case["op"] == "linear":
        K, N, g = case["K"], case["N"], 2 if case["glu"] else 1
        b = (t * K + g * N * K) * e + t * N * es[case["out"]] + 4 * N * (g * case["bias"] + rows[case["gate"]])
        return {"bytes": b + (0 if case["res"] == "none" else t * N * es[case["res"]]), "flops": 2 * t * K * N * g}
    H, D, past = case["H"], case["D"], case["past"]
    if case["op"] == "append":
        return {"bytes": 4 * t * H * D * e, "flops": 0}
    w, S = case["window"], case["sinks"]
    if w:
        S = min(S, past)
        keys = min(S + w + n, past + n)
        seen = n * min(S + w, past + n) if case["causal"] else n * keys
    else:
        keys = past + n
        seen = n * past + (n * (n + 1) // 2 if case["causal"] else n * n)
    return {"bytes": 2 * t * case["Hq"] * D * e + 2 * B * H * keys * D * e, "flops": 4 * B * case["Hq"] * seen * D}


# ------------------------------------------------------------------- exact

def _exact_norm(x, kind, gain, bias):
    if kind == "none":
        return x
    C = x.shape[-1]
    if kind == "layer":
        x = x - (x.sum(-1) / C)[..., None]
    x = x / ((x * x).sum(-1) / C + EPS).sqrt()[..., None] * gain.double()
    return x + bias.double() if bias is not None else x


def _exact_act(x, act):
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "gelu":   # (1 + tanh z) / 2 = 1 / (1 + exp(-2 z))
        return x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return x


def _behind(out, lens):
    """Rows behind an entry's last token, as they were."""
    for b, m in enumerate(lens):
        for o in out:
            if o is not None:
                o[b, m:] = 0
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    lens, B, n = s["lens"].tolist(), case["B"], case["n"]
    if case["op"] == "norm":
        r = s["x"].double() * case["xs"]
        if case["h"]:
            h = _exact_norm(s["h"].double(), case["post"], s["post_gain"], s["post_bias"])
            r += h * (1.0 if s["gate"] is None else s["gate"].double())
        y = None
        if case["pre"] != "none":
            y = _exact_norm(r, case["pre"], s["pre_gain"], s["pre_bias"])
            if s["scale"] is not None:
                y = y + y * s["scale"].double() + s["shift"].double()
        return tuple(_behind([r if case["h"] else None, y], lens))
    if case["op"] == "linear":
        N = case["N"]
        out = torch.empty(B, n, N, device="cuda", dtype=torch.float64)
        w = s["w"].double()
        for b in range(B):
            z = s["x"][b].double() @ w.t()
            if case["bias"]:
                z += s["bias"].double()
            z = _exact_act(z[:, :N], case["act"]) * (z[:, N:] if case["glu"] else 1.0)
            if s["gate"] is not None:
                z *= s["gate"].double().expand(B, n, N)[b]
            out[b] = z if s["res"] is None else z + s["res"][b].double()
        return _behind([out], lens)[0]
    pos, table, ps = s["pos"].tolist(), s["table"].tolist(), case["ps"]
    if case["op"] == "append":
        out = [p.double() for p in s["pool"]]
        for b in range(B):
            i = 0
            while i < lens[b]:   # a page's tokens at a time
                page, off = table[b][(pos[b] + i) // ps], (pos[b] + i) % ps
                m = min(ps - off, lens[b] - i)
                for o, x in zip(out, (s["k"], s["v"])):
                    o[page, off:off + m] = x[b, i:i + m].double()
                i += m
        return tuple(out)
    # one entry and key head after the other, over the visible positions in order
    S, w, H, g, D = case["sinks"], case["window"], case["H"], case["Hq"] // case["H"], case["D"]
    out = torch.zeros(B, n, case["Hq"], D, device="cuda", dtype=torch.float64)
    for b in range(B):
        m = lens[b]
        if m == 0:
            continue
        low = 0 if not w else max(0, pos[b] - w)
        at = torch.tensor([j for j in range(pos[b] + m) if j < S or j >= low], device="cuda")
        mine = (pos[b] + torch.arange(m, device="cuda"))[:, None]
        bar = torch.zeros(m, len(at), device="cuda", dtype=torch.float64)
        if case["causal"]:
            bar[at > mine] = -math.inf
            if w:
                bar[(at >= S) & (at <= mine - w)] = -math.inf
        page = s["table"][b].long()[at // ps]
        for h in range(H):
            k, v = (p[page, at % ps, h].double() for p in s["pool"])
            q = s["q"][b, :m, h * g:(h + 1) * g].double().permute(1, 0, 2)
            p = torch.softmax(torch.matmul(q, k.t()) / math.sqrt(D) + bar, -1)
            out[b, :m, h * g:(h + 1) * g] = torch.matmul(p, v).permute(1, 0, 2)
    return out
