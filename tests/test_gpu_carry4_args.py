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
