"""Arguments of the Python calls of a block's operators that the C calls would
misread, or whose results would overlap: DcError, nothing is launched."""
import pytest

from paper_2609_35115_amd import DcError

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def refuse(match, f, *a, **k):
    with pytest.raises(DcError, match=match):
        f(*a, **k)


def test_norm_residual_refusals():
    from paper_2609_35115_amd.block import Norm, norm_residual as f
    z = lambda *s, dt=torch.float32: torch.zeros(*s, device="cuda", dtype=dt)   # noqa: E731
    x, h = z(2, 3, 64), z(2, 3, 64, dt=torch.bfloat16)
    pre = Norm("rms", z(64))
    refuse("GPU", f, torch.zeros(2, 3, 64), pre=pre)
    refuse("three dimensions", f, z(3, 64), pre=pre)
    refuse("h must be", f, x, z(2, 3, 65), pre=pre)
    refuse("on cuda", f, x, torch.zeros(2, 3, 64), pre=pre)
    refuse("float32 or bfloat16", f, x, z(2, 3, 64, dt=torch.float16), pre=pre)
    refuse("consecutive", f, x, z(2, 64, 3).transpose(1, 2), pre=pre)
    refuse("weights must be", f, x, h, pre=Norm("rms", z(65)))
    refuse("kind", Norm, "batch")
    refuse("gain", Norm, "rms", z(64, dt=torch.bfloat16))
    refuse("bias", Norm, "rms", z(64), z(65))
    refuse("nothing to compute", f, x)
    refuse("go with h", f, x, pre=pre, gate=z(64))
    refuse("go with y", f, x, h, pre=pre, out=(x, None))
    refuse("finite", f, x, h, x_scale=float("inf"))
    refuse("eps", f, x, h, pre=Norm("rms", eps=-1.0))
    for bad in (z(65), z(3, 64), z(2, 2, 64), z(1, 2, 3, 64), torch.zeros(64)):
        refuse("gate", f, x, h, gate=bad)
    refuse("lens", f, x, h, lens=torch.zeros(2, device="cuda", dtype=torch.int64))
    refuse("lens", f, x, h, lens=torch.zeros(3, device="cuda", dtype=torch.int32))
    # results
    refuse("out\\[0\\] must be torch.float32", f, x, h, out=(z(2, 3, 64, dt=torch.bfloat16), None))
    refuse("out\\[1\\] must be torch.bfloat16", f, x, h, pre=pre, out=(None, z(2, 3, 64)))
    y = torch.zeros_like(h)
    for over in (z(1, 3, 64).expand(2, 3, 64), z(2, 1, 64).expand(2, 3, 64), z(400).as_strided((2, 3, 64), (192, 63, 1)),
                 z(400).as_strided((2, 3, 64), (64, 64, 1))):
        refuse("overlap", f, x, h, out=(over, None))
    refuse("overlap", f, x, x, pre=pre, out=(x, x))
    big = z(2, 6, 64)
    refuse("overlap", f, big[:, ::2], h, out=(big[:, :3], None))
    refuse("overlap", f, x, big[:, ::2], pre=pre, out=(None, big[:, :3]))
    # two dimensions with one row each are no overlap, and neither is a call of no tokens
    f(x[:1, :1], h[:1, :1], out=(z(1, 1, 64).as_strided((1, 1, 64), (0, 0, 1)), None))
    r, y = f(x[:, :0], h[:, :0], pre=pre)
    assert r.shape == y.shape == (2, 0, 64)
    assert f(x, h, pre=pre, out=(None, torch.zeros_like(h)))[0] is None


def test_linear_refusals():
    from paper_2609_35115_amd.block import linear as f
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, device="cuda", dtype=dt)   # noqa: E731
    x, w = z(2, 3, 64), z(48, 64)
    refuse("act", f, x, w, act="relu")
    refuse("weight must be", f, x, z(48, 63))
    refuse("weight must be", f, x, z(48, 64, dt=torch.float32))
    refuse("weight must be", f, x, torch.zeros(48, 64, dtype=torch.bfloat16))
    refuse("consecutive", f, x, z(64, 48).t())
    refuse("even", f, x, z(47, 64), act="silu_glu")
    refuse("bias", f, x, w, z(48))
    refuse("bias", f, x, w, z(24, dt=torch.float32))
    refuse("residual must be", f, x, w, residual=z(2, 3, 47))
    refuse("gate", f, x, w, gate=z(47))
    refuse("finite", f, x, w, residual=z(2, 3, 48), residual_scale=float("nan"))
    refuse("out must be", f, x, w, out=z(2, 3, 47))
    refuse("out must be", f, x, w, out=z(2, 3, 48), out_dtype=torch.float32)
    refuse("float32 or bfloat16", f, x, w, out_dtype=torch.float16)
    refuse("overlap", f, x, w, out=z(2, 1, 48).expand(2, 3, 48))
    refuse("overlap", f, x, z(64, 64), out=x)
    buf = z(2, 6, 48)
    refuse("overlap", f, x, w, residual=buf[:, :3], out=buf[:, ::2])
    refuse("stride", f, x, z(1, 64).expand(48, 64))
    assert f(x[:, :0], w).shape == (2, 0, 48)


def test_paged_refusals():
    from paper_2609_35115_amd.paged import PagedCarry
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, device="cuda", dtype=dt)   # noqa: E731
    i = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.int32)             # noqa: E731
    k = z(5, 16, 2, 64)
    refuse("type, device and shape", PagedCarry, k, z(5, 16, 2, 128), i(2, 2))
    refuse("type, device and shape", PagedCarry, k, z(5, 16, 2, 64, dt=torch.float32), i(2, 2))
    refuse("four dimensions", PagedCarry, z(5, 16, 128), z(5, 16, 128), i(2, 2))
    refuse("table must be", PagedCarry, k, k.clone(), i(2, 2).long())
    refuse("table must be", PagedCarry, k, k.clone(), i(2))
    refuse("table must be", PagedCarry, k, k.clone(), torch.zeros(2, 2, dtype=torch.int32))
    refuse("power of two", PagedCarry, z(5, 12, 2, 64), z(5, 12, 2, 64), i(2, 2))
    refuse("head_dim", PagedCarry, z(5, 16, 2, 32), z(5, 16, 2, 32), i(2, 2))
    refuse("16 bytes", PagedCarry, z(5, 16, 2, 65)[..., 1:], k, i(2, 2))
    refuse("overlap", PagedCarry, z(1, 16, 2, 64).expand(5, 16, 2, 64), k, i(2, 2))
    refuse("float32 or bfloat16", PagedCarry, k.half(), k.half(), i(2, 2))
    c = PagedCarry(k, k.clone(), i(2, 2))
    pos = torch.zeros(2, device="cuda", dtype=torch.int64)
    a, q = z(2, 3, 2, 64), z(2, 3, 4, 64)
    refuse("k must be", c.append, a.float(), a, pos)
    refuse("v must be", c.append, a, z(2, 3, 1, 64), pos)
    refuse("pos", c.append, a, a, pos.int())
    refuse("pos", c.append, a, a, None)
    refuse("lens", c.append, a, a, pos, lens=pos)
    refuse("multiple", c.attend, z(2, 3, 3, 64), pos)
    refuse("four dimensions", c.attend, z(2, 3, 256), pos)
    refuse("window", c.attend, q, pos, window=0)
    refuse("window", c.attend, q, pos, window=2 ** 31)
    refuse("sinks", c.attend, q, pos, window=4, sinks=-1)
    refuse("finite", c.attend, q, pos, scale=float("nan"))
    refuse("overlap", c.attend, q, pos, out=z(2, 1, 4, 64).expand(2, 3, 4, 64))
    buf = z(2, 6, 4, 64)
    refuse("overlap", c.attend, buf[:, ::2], pos, out=buf[:, :3])
    long = a[:, :1].expand(2, 2 ** 32 + 1, 2, 64)
    refuse("2\\^31", c.append, long, long, pos)
    refuse("2\\^31", c.attend, long, pos)
    assert c.attend(q[:, :0], pos).shape == (2, 0, 4, 64)
    assert not bool(k.any())
