"""The attention operators' C calls on the host: sizes, and every refusal
before anything is launched (CPU; the pointers are never read)."""
import ctypes
from ctypes import byref

import pytest

import paper_2609_35115_amd as dc
from paper_2609_35115_amd import flow

L = flow.flib()
P = 1 << 20   # an address that is only looked at


def carry(**k):
    c = dict(abi_version=1, batch=2, heads=2, head_dim=64, sinks=3, ring=8, data=P)
    c.update(k)
    return flow.DcCarry4(*c.values())


def span(**k):
    s = dict(pos=P, lens=None, sinks=None, batch=2, n=4)
    s.update(k)
    return flow.DcSpan(*s.values())


def rows(heads=2, data=P):
    return flow.DcHeadRows(data, 4 * heads * 64, heads * 64, 64, heads)


def norm(**k):
    m = dict(q_gain=None, k_gain=None, freqs=P, n_freqs=32, interleaved=0, eps=1e-6)
    m.update(k)
    return flow.DcQkNorm(*m.values())


def ref(x):
    return None if x is None else byref(x)


def append(c=carry(), m=None, s=span(), dtype=1, q=None, k=rows(), v=rows(), o=None):
    return L.dc_carry4_append(ref(c), ref(m), ref(s), dtype, ref(q), ref(k), ref(v), ref(o), None)


def attend(c=carry(), s=span(), dtype=1, q=rows(4), o=rows(4), window=3, causal=1, scale=0.1, ws=None, size=0):
    return L.dc_carry4_attend(ref(c), ref(s), dtype, ref(q), ref(o), window, causal, scale, ws, size, None)


def rotate(m=norm(), s=span(), D=64, dtype=1, q=rows(4), k=rows(), qo=rows(4), ko=rows()):
    return L.dc_qk_norm_rope(ref(m), ref(s), D, dtype, ref(q), ref(k), ref(qo), ref(ko), None)


def test_struct_sizes_match_header_layout():
    assert ctypes.sizeof(flow.DcCarry4) == 6 * 4 + 8
    assert ctypes.sizeof(flow.DcSpan) == 3 * 8 + 2 * 4
    assert ctypes.sizeof(flow.DcHeadRows) == 4 * 8 + 8
    assert ctypes.sizeof(flow.DcQkNorm) == 3 * 8 + 2 * 4 + 8


def test_carry_bytes():
    for heads, D, slots in ((2, 64, 11), (1, 128, 458), (8, 64, 1 << 20)):
        c = carry(batch=3, heads=heads, head_dim=D, sinks=2, ring=slots - 2)
        region = (slots * (D + D // 16) + 255) // 256 * 256   # codes and scales of keys and values: 4.25 bits each
        assert L.dc_carry4_bytes(byref(c)) == 3 * heads * region
    assert L.dc_carry4_bytes(byref(carry(data=None))) > 0
    for bad in (dict(abi_version=2), dict(batch=0), dict(heads=0), dict(head_dim=32), dict(sinks=-1), dict(ring=0),
                dict(ring=1 << 24)):
        assert L.dc_carry4_bytes(byref(carry(**bad))) == 0
    assert L.dc_carry4_bytes(None) == 0


def test_workspace():
    assert L.dc_carry4_workspace(byref(carry()), 4, 4, 3) == 0                   # a short carry is not split
    long = carry(ring=100_000)
    size = L.dc_carry4_workspace(byref(long), 4, 1, 99_999)
    assert size > 0 and size % (2 * 4 * 66 * 4) == 0                             # whole rows of results, maximum, sum
    assert attend(c=long, s=span(n=1), window=99_999) == dc.DC_EINVAL            # without one
    assert b"workspace" in L.dc_carry4_last_error()
    assert attend(c=long, s=span(n=1), window=99_999, ws=P, size=size - 1) == dc.DC_EINVAL
    assert attend(c=long, s=span(n=1), window=99_999, ws=P + 4, size=size) == dc.DC_EINVAL
    for args in ((3, 1, 5), (0, 1, 5), (4, 0, 5), (4, 1, -1)):
        assert L.dc_carry4_workspace(byref(long), *args) == 0


@pytest.mark.parametrize("call", [append, attend])
def test_carry_and_span_refusals(call):
    bad = [dict(c=None), dict(s=None), dict(c=carry(data=None)), dict(c=carry(data=P + 16)), dict(c=carry(batch=3)),
           dict(s=span(pos=None)), dict(s=span(batch=0)), dict(s=span(n=-1)), dict(dtype=2), dict(c=carry(head_dim=96)),
           dict(c=carry(sinks=-1)), dict(c=carry(ring=0))]
    for k in bad:
        assert call(**k) == dc.DC_EINVAL, k
        assert L.dc_carry4_last_error()
    assert call(c=carry(abi_version=0)) == dc.DC_EVERSION
    assert call(c=carry(ring=1 << 24)) == dc.DC_ERANGE
    assert call(c=carry(ring=(1 << 24) - 3), s=span(n=(1 << 31) - 1)) in (dc.DC_ERANGE,)


def test_append_refusals():
    for k in (dict(k=None), dict(v=None), dict(k=rows(1)), dict(v=rows(3)), dict(k=rows(data=None)), dict(k=rows(data=P + 1)),
              dict(q=rows(4)), dict(o=rows(4)), dict(m=norm()), dict(m=norm(), q=rows(4)), dict(m=norm(), q=rows(4), o=rows(2)),
              dict(m=norm(n_freqs=4), q=rows(4), o=rows(4)), dict(m=norm(freqs=None), q=rows(4), o=rows(4))):
        assert append(**k) == dc.DC_EINVAL, k


def test_attend_refusals():
    for k in (dict(q=None), dict(o=None), dict(q=rows(3), o=rows(3)), dict(o=rows(2)), dict(window=0), dict(window=-1, causal=0),
              dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(**k) == dc.DC_EINVAL, k
    for k in (dict(window=9), dict(window=8, causal=0), dict(window=(1 << 31) - 1)):   # 4 tokens, 3 + 8 slots
        assert attend(**k) == dc.DC_ERANGE, k
    assert b"carry" in L.dc_carry4_last_error()


def test_norm_refusals():
    for k in (dict(m=None), dict(s=None), dict(D=32), dict(dtype=-1), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None),
              dict(qo=rows(3)), dict(ko=rows(1)), dict(m=norm(n_freqs=4)), dict(m=norm(n_freqs=40)), dict(m=norm(n_freqs=-8)),
              dict(m=norm(freqs=None)), dict(m=norm(eps=-1.0)), dict(m=norm(eps=float("nan")))):
        assert rotate(**k) == dc.DC_EINVAL, k
    assert rotate(s=span(n=(1 << 31) - 1)) == dc.DC_ERANGE


def test_a_call_of_no_tokens_launches_nothing():
    none = rows(data=None)
    s = span(n=0)
    assert append(s=s, k=none, v=none) == dc.DC_OK
    assert attend(s=s, q=rows(4, None), o=rows(4, None)) == dc.DC_OK
    assert rotate(s=s, q=rows(4, None), k=none, qo=rows(4, None), ko=none) == dc.DC_OK
