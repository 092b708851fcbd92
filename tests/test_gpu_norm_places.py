"""One result of a norm in an input's place, the other elsewhere (GPU): the same bits
as with both apart, at widths whose last vector repeats elements of another wave's."""
from __future__ import annotations

import itertools

import pytest

from tests.gpu_common import say

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("width", [5, 63, 517, 1025, 1027, 1031, 1539, 2051, 2571, 4097, 9001, 16383])
def test_one_result_in_place(width, dtype):
    from paper_2609_35115_amd.block import Norm, norm_residual
    g = torch.Generator(device="cuda").manual_seed(width)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    B, n = 3, 900 if width < 4000 else 150
    x, h = rand(B, n, width).to(dtype), rand(B, n, width).to(dtype)
    scale, shift, token = rand(width), rand(B, width), rand(B, n, width)
    lens = torch.tensor([n, 0, n // 2], device="cuda", dtype=torch.int32)
    rows = torch.arange(n, device="cuda") < lens[:, None]
    for k in (dict(), dict(scale=scale, shift=shift), dict(pre=Norm("layer")), dict(pre=Norm("rms"), scale=token), dict(post=Norm("rms")),
              dict(post=Norm("layer"), pre=Norm("rms"))):
        say(f"norm {width} {dtype} {sorted(k)}")
        want = norm_residual(x, h, x_scale=0.5, out=(torch.empty_like(x), torch.empty_like(h)), **k)
        for r, y in itertools.product(("x", "h", "r", None), ("x", "h", "y", None)):
            if r == y or (y is None and ("pre" in k or "scale" in k)):
                continue
            for some in (None, lens):
                at = {"x": x.clone(), "h": h.clone(), "r": torch.full_like(x, 7.0), "y": torch.full_like(h, 7.0), None: None}
                old = {name: t.clone() for name, t in at.items() if t is not None}
                got = norm_residual(at["x"], at["h"], x_scale=0.5, lens=some, out=(at[r], at[y]), **k)
                for name, o, w in zip((r, y), got, want):
                    if o is None:
                        continue
                    assert torch.equal(o if some is None else o[rows], w if some is None else w[rows]), (r, y, sorted(k))
                    assert some is None or torch.equal(o[~rows], old[name][~rows])
                for name, t in old.items():   # what is no result is as it was
                    assert name in (r, y) or torch.equal(at[name], t)


@pytest.mark.parametrize("width", [517, 1025, 2051, 4097])
def test_the_norm_of_x_in_its_place(width):
    from paper_2609_35115_amd.block import Norm, norm_residual
    g = torch.Generator(device="cuda").manual_seed(width)
    x = torch.randn(2, 700, width, generator=g, device="cuda")
    for k in (dict(pre=Norm("rms")), dict(scale=torch.randn(width, generator=g, device="cuda"))):
        want = norm_residual(x, x_scale=2.0, out=(torch.empty_like(x), torch.empty_like(x)), **k)
        for which in (0, 1):
            a = x.clone()
            out = [torch.empty_like(x), torch.empty_like(x)]
            out[which] = a
            got = norm_residual(a, x_scale=2.0, out=tuple(out), **k)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        a = x.clone()
        assert torch.equal(norm_residual(a, x_scale=2.0, out=(None, a), **k)[1], want[1])
