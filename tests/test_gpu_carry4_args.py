"""Arguments of the Python calls that do not fit the C structures: DcError, and
nothing is launched or allocated."""
import pytest
import torch

from paper_2609_35115_amd import DcError
from tests.test_gpu_carry4 import carry4, index, rand

pytestmark = pytest.mark.gpu


def test_sizes_that_do_not_fit_their_fields():
    m = carry4()
    c = m.Carry4(2, 2, 64, sinks=1, ring=8)
    c.memory.fill_(17)
    k, pos, f = rand((2, 1, 2, 64), "bf16", 1), index([0, 0]), torch.ones(8, device="cuda")
    long, wide = k.expand(2, 2 ** 32 + 1, 2, 64), k[:, :, :1].expand(2, 1, 2 ** 32 + 2, 64)
    free = torch.cuda.memory_allocated()
    for call in (lambda: c.append(long, long, pos), lambda: c.append_rotated(long, long, long, pos, f),
                 lambda: c.append_rotated(wide, k, k, pos, f), lambda: c.attend(long, pos, 1), lambda: c.attend(wide, pos, 1),
                 lambda: m.qk_norm_rope(long, long, pos, f), lambda: m.qk_norm_rope(wide, k, pos, f),
                 lambda: m.qk_norm_rope(k, wide, pos, f)):
        with pytest.raises(DcError, match="2\\^31"):
            call()
    for eps in (1e39, -1e39):
        with pytest.raises(DcError, match="eps"):
            m.qk_norm_rope(k, k, pos, f, eps=eps)
        with pytest.raises(DcError, match="eps"):
            c.append_rotated(k, k, k, pos, f, eps=eps)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == free and (c.memory == 17).all()


def test_results_that_overlap():
    """A result with one place for several rows, and results over each other's inputs:
    refused, nothing is written."""
    m = carry4()
    c = m.Carry4(2, 2, 64, sinks=1, ring=8)
    k, pos, f = rand((2, 3, 2, 64), "bf16", 1), index([0, 0]), torch.ones(8, device="cuda")
    q, keep = k.clone(), k.clone()
    c.append(k, k, pos)
    fresh = lambda: torch.zeros_like(k)
    for shape in ((1, 3, 2, 64), (2, 1, 2, 64), (2, 3, 1, 64)):
        one = torch.zeros(shape, dtype=k.dtype, device="cuda")
        over = one.expand(2, 3, 2, 64)
        for call in (lambda: c.attend(q, pos, 4, out=over), lambda: c.append_rotated(q, k, k, pos, f, out=over),
                     lambda: m.qk_norm_rope(q, k, pos, f, out=(over, fresh())), lambda: m.qk_norm_rope(q, k, pos, f, out=(fresh(), over))):
            with pytest.raises(DcError, match="overlap"):
                call()
        assert not one.any()
    for out in ((k, fresh()), (fresh(), q), (k, q), (k, k)):
        with pytest.raises(DcError, match="overlap"):
            m.qk_norm_rope(q, k, pos, f, out=out)
    one = fresh()
    with pytest.raises(DcError, match="overlap"):
        m.qk_norm_rope(q, k, pos, f, out=(one, one))
    with pytest.raises(DcError, match="overlap"):
        c.append_rotated(q, k, k.clone(), pos, f, out=k)
    with pytest.raises(DcError, match="overlap"):
        c.append_rotated(q, k.clone(), k, pos, f, out=k)
    assert torch.equal(k, keep) and torch.equal(q, keep)
    # broadcast inputs, and a single row of stride 0, are no overlap
    a, b = m.qk_norm_rope(q[:1].expand(2, 3, 2, 64), k, pos, f)
    assert torch.equal(a[0], a[1])
    single = torch.zeros(1, 1, 1, 64, dtype=k.dtype, device="cuda").as_strided((1, 1, 1, 64), (0, 0, 0, 1))
    d = m.Carry4(1, 1, 64, sinks=0, ring=2)
    d.append(k[:1, :1, :1], k[:1, :1, :1], pos[:1])
    assert d.attend(q[:1, :1, :1], pos[:1], 1, out=single) is single and single.any()
    # nor is a call of no tokens
    a, b = m.qk_norm_rope(q[:, :0], k[:, :0], pos, f, out=(k[:, :0], k[:, :0]))
    assert a.shape == (2, 0, 2, 64)
