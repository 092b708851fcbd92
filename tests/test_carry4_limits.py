"""The attention operators' sizes at and past their limits: refused with DC_ERANGE
before anything is launched (CPU; the pointers are never read)."""
from ctypes import byref

import pytest

import paper_2609_35115_amd as dc
from tests.test_carry4_args import L, append, attend, carry, norm, ref, rotate, rows, span


def read(c=carry(), s=span(), dtype=1, k=rows(), v=rows()):
    return L.dc_carry4_read(ref(c), ref(s), dtype, ref(k), ref(v), None)


@pytest.mark.parametrize("q,k,batch,n", [
    (1 << 29, 1 << 29, 1 << 20, 1 << 14),     # 2^64 rows, 0 in 64 bits
    (1 << 30, 1 << 30, 1 << 30, 1 << 30),
    ((1 << 31) - 1, (1 << 31) - 1, (1 << 31) - 1, (1 << 31) - 1),
    (3, 1, 1 << 30, 1 << 30),
    (1 << 30, 1, 1, 1), (1, 1, 1 << 30, 1), (1, 1, 1, 1 << 30),   # just past
])
@pytest.mark.parametrize("D", [64, 128])
def test_products_of_sizes_past_64_bits(q, k, batch, n, D):
    s = span(batch=batch, n=n)
    assert rotate(s=s, D=D, q=rows(q), k=rows(k), qo=rows(q), ko=rows(k)) == dc.DC_ERANGE
    assert b"too many rows" in L.dc_carry4_last_error()
    if batch * k <= 1 << 26:
        c = carry(batch=batch, heads=k, head_dim=D, ring=(1 << 24) - 3)
        assert append(c=c, s=s, m=norm(), q=rows(q), o=rows(q), k=rows(k), v=rows(k)) == dc.DC_ERANGE
        if q * batch * n > 1 << 30:
            assert attend(c=c, s=s, q=rows(q // k * k), o=rows(q // k * k), window=1) == dc.DC_ERANGE


@pytest.mark.parametrize("k,n", [(1 << 20, 1 << 30), (1, (1 << 31) - 1), (1 << 6, 1 << 24)])
def test_stores_and_reads_past_the_limit(k, n):
    c, s = carry(batch=64, heads=k), span(batch=64, n=n)
    assert append(c=c, s=s, k=rows(k), v=rows(k)) == dc.DC_ERANGE
    assert read(c=c, s=s, k=rows(k), v=rows(k)) == dc.DC_ERANGE


@pytest.mark.parametrize("q_heads,n", [(1 << 30, (1 << 31) - 1), (1 << 30, 1), (4, (1 << 31) - 1), ((1 << 31) - 2, 1 << 30)])
@pytest.mark.parametrize("c", [carry(ring=(1 << 24) - 3), carry(batch=1 << 20, heads=1 << 1, head_dim=128)])
def test_no_workspace_for_a_call_past_the_limit(c, q_heads, n):
    assert L.dc_carry4_workspace(byref(c), q_heads, n, 1 << 20) == 0


# A launch has fewer than 2^24 blocks of 256 threads.

@pytest.mark.parametrize("batch,heads,q", [(1 << 21, 8, 8), (1 << 23, 8, 16), (1 << 24, 4, 4)])
def test_attention_of_more_regions_than_a_launch_has_blocks(batch, heads, q):
    c = carry(batch=batch, heads=heads, sinks=0)
    assert attend(c=c, s=span(batch=batch, n=1), q=rows(q), o=rows(q)) == dc.DC_ERANGE
    assert b"too many rows" in L.dc_carry4_last_error()


@pytest.mark.parametrize("D,n", [(64, 1 << 15), (128, 1 << 14)])
def test_norms_and_stores_of_more_tokens_than_a_launch_has_blocks(D, n):
    one, s = rows(1), span(batch=1 << 14, n=n)
    assert rotate(s=s, D=D, q=one, k=one, qo=one, ko=one) == dc.DC_ERANGE
    c = carry(batch=1 << 14, heads=1, head_dim=D)
    assert append(c=c, s=s, k=one, v=one) == dc.DC_ERANGE
    assert read(c=c, s=s, k=one, v=one) == dc.DC_ERANGE
    assert b"too many rows" in L.dc_carry4_last_error()


def test_scales_whose_product_with_log2_e_is_infinite():
    """(A score of zero times it would be NaN.)"""
    for scale in (3e38, -3e38, 2.3588e38):
        assert attend(scale=scale) == dc.DC_EINVAL
        assert b"scale" in L.dc_carry4_last_error()
    none = rows(4, None)
    assert attend(s=span(n=0), q=none, o=none, scale=2.3586e38) == dc.DC_OK
