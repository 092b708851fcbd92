"""The C calls of a block's operators on the host: sizes, and every refusal
before anything is launched (CPU; the pointers are never read)."""
import ctypes
from ctypes import byref

import pytest

import paper_2609_35115_amd as dc
from paper_2609_35115_amd import flow

L = flow.flib()
P = 1 << 20   # an address that is only looked at
MAX = (1 << 31) - 1


def call(**k):
    c = dict(lens=None, batch=2, n=3)
    c.update(k)
    return flow.DcCall(*c.values())


def rows(dtype=1, data=P, sb=3 * 64, st=64):
    return flow.DcRows(data, sb, st, dtype)


def norm(**k):
    m = dict(kind=1, eps=1e-6, gain=P, bias=None)
    m.update(k)
    return flow.DcNorm(*m.values())


def layer(**k):
    m = dict(weight=P, bias=None, stride=64, n_in=64, n_out=48, dtype=1, act=0, glu=0)
    m.update(k)
    return flow.DcLinearLayer(*m.values())


def paged(**k):
    c = dict(abi_version=1, batch=2, heads=2, head_dim=64, dtype=1, page_size=16, pages=9, table_pages=4, table=P, table_stride=4, k=P, v=P,
             k_stride_page=2048, k_stride_t=128, k_stride_h=64, v_stride_page=2048, v_stride_t=128, v_stride_h=64)
    c.update(k)
    return flow.DcPaged(*c.values())


def span(**k):
    s = dict(pos=P, lens=None, sinks=None, batch=2, n=3)
    s.update(k)
    return flow.DcSpan(*s.values())


def heads(h=2, data=P):
    return flow.DcHeadRows(data, 4 * h * 64, h * 64, 64, h)


def ref(x):
    return None if x is None else byref(x)


def residual(c=call(), width=64, x=rows(), xs=1.0, h=rows(), post=None, gate=None, r=rows(), pre=None, scale=None, shift=None, y=None):
    return L.dc_norm_residual(ref(c), width, ref(x), xs, ref(h), ref(post), ref(gate), ref(r), ref(pre), ref(scale), ref(shift), ref(y), None)


def linear(c=call(), m=layer(), x=rows(), gate=None, res=None, rs=1.0, out=rows(), ws=None, size=0):
    return L.dc_linear(ref(c), ref(m), ref(x), ref(gate), ref(res), rs, ref(out), ws, size, None)


def append(c=paged(), s=span(), k=heads(), v=heads()):
    return L.dc_paged_append(ref(c), ref(s), ref(k), ref(v), None)


def attend(c=paged(), s=span(), q=heads(4), o=heads(4), window=0, sinks=0, causal=1, scale=0.1, ws=None, size=0):
    return L.dc_paged_attend(ref(c), ref(s), ref(q), ref(o), window, sinks, causal, scale, ws, size, None)


def test_struct_sizes_match_header_layout():
    assert ctypes.sizeof(flow.DcCall) == 8 + 2 * 4
    assert ctypes.sizeof(flow.DcRows) == 3 * 8 + 8
    assert ctypes.sizeof(flow.DcNorm) == 2 * 4 + 2 * 8
    assert ctypes.sizeof(flow.DcLinearLayer) == 3 * 8 + 5 * 4 + 4
    assert ctypes.sizeof(flow.DcPaged) == 8 * 4 + 4 * 8 + 6 * 8


def test_norm_refusals():
    nan, inf = float("nan"), float("inf")
    for k in (dict(c=None), dict(c=call(batch=0)), dict(c=call(n=-1)), dict(width=0), dict(width=-5), dict(x=None), dict(x=rows(data=None)),
              dict(x=rows(data=P + 1)), dict(x=rows(dtype=2)), dict(xs=nan), dict(xs=inf), dict(r=None), dict(h=None, post=norm()),
              dict(h=None, gate=rows()), dict(pre=norm()), dict(scale=rows()), dict(shift=rows()), dict(post=norm(kind=0)), dict(post=norm(kind=3)),
              dict(post=norm(eps=-1.0)), dict(post=norm(eps=nan)), dict(post=norm(gain=P + 2)), dict(y=rows(), pre=norm(bias=P + 1)),
              dict(gate=rows(dtype=7)), dict(gate=rows(data=None)), dict(r=rows(dtype=0)), dict(r=rows(sb=0)), dict(r=rows(st=0)),
              dict(y=rows(dtype=0)), dict(y=rows(sb=0)), dict(h=rows(dtype=0, data=P + 2))):
        assert residual(**k) == dc.DC_EINVAL, k
        assert L.dc_block_last_error()
    for k in (dict(width=16385), dict(c=call(n=MAX)), dict(c=call(batch=MAX, n=MAX))):
        assert residual(**k) == dc.DC_ERANGE, k


def test_linear_refusals():
    for k in (dict(c=None), dict(c=call(batch=-1)), dict(m=None), dict(m=layer(weight=None)), dict(m=layer(weight=P + 1)), dict(m=layer(bias=P + 2)),
              dict(m=layer(stride=63)), dict(m=layer(n_in=0)), dict(m=layer(n_out=0)), dict(m=layer(dtype=3)), dict(m=layer(act=3)),
              dict(m=layer(act=-1)), dict(x=None), dict(x=rows(dtype=0)), dict(out=None), dict(out=rows(dtype=5)), dict(out=rows(st=0)),
              dict(gate=rows(dtype=9)), dict(res=rows(data=None)), dict(rs=float("inf"))):
        assert linear(**k) == dc.DC_EINVAL, k
        assert L.dc_block_last_error()
    for k in (dict(m=layer(n_in=(1 << 24) + 1, stride=1 << 25)), dict(m=layer(n_out=(1 << 24) + 1)), dict(c=call(n=MAX))):
        assert linear(**k) == dc.DC_ERANGE, k


def test_linear_workspace():
    assert L.dc_linear_workspace(byref(layer()), 2, 3) == 0                     # a short sum is not split
    long = layer(n_in=8192, stride=8192, n_out=64)
    size = L.dc_linear_workspace(byref(long), 1, 4)
    assert size > 0 and size % (4 * 64 * 4) == 0                                # whole rows of partial sums
    x = rows(sb=8192, st=8192)
    assert linear(c=call(batch=1, n=4), m=long, x=x) == dc.DC_EINVAL            # without one
    assert b"workspace" in L.dc_block_last_error()
    assert linear(c=call(batch=1, n=4), m=long, x=x, ws=P, size=size - 1) == dc.DC_EINVAL
    assert linear(c=call(batch=1, n=4), m=long, x=x, ws=P + 8, size=size) == dc.DC_EINVAL
    for m, b, n in ((layer(n_in=0), 1, 4), (long, 0, 4), (long, 1, 0), (long, 1, -1), (long, MAX, MAX)):
        assert L.dc_linear_workspace(byref(m), b, n) == 0
    assert L.dc_linear_workspace(None, 1, 1) == 0


@pytest.mark.parametrize("f", [append, attend])
def test_cache_and_span_refusals(f):
    for k in (dict(batch=0), dict(heads=0), dict(head_dim=96), dict(dtype=2), dict(page_size=0), dict(page_size=24), dict(page_size=-16),
              dict(page_size=-(1 << 31)), dict(pages=0), dict(table_pages=0), dict(table=None), dict(table=P + 2), dict(k=None), dict(v=P + 8),
              dict(k_stride_t=60), dict(v_stride_h=4), dict(k_stride_page=-2048), dict(v_stride_page=2047)):
        assert f(c=paged(**k)) == dc.DC_EINVAL, k
        assert L.dc_block_last_error()
    assert f(c=None) == dc.DC_EINVAL and f(c=paged(abi_version=2)) == dc.DC_EVERSION
    for k in (dict(table_pages=1 << 27), dict(page_size=1 << 30, table_pages=2), dict(batch=1 << 20, heads=1 << 20), dict(k_stride_page=1 << 36)):
        assert f(c=paged(**k)) == dc.DC_ERANGE, k
    for k in (dict(pos=None), dict(batch=3), dict(n=-1)):
        assert f(s=span(**k)) == dc.DC_EINVAL, k
    assert f(s=None) == dc.DC_EINVAL and f(s=span(n=MAX)) == dc.DC_ERANGE


def test_append_refusals():
    for k in (dict(k=None), dict(v=None), dict(k=heads(1)), dict(v=heads(3)), dict(k=heads(data=None)), dict(v=heads(data=P + 1))):
        assert append(**k) == dc.DC_EINVAL, k


def test_attend_refusals():
    for k in (dict(q=None), dict(o=None), dict(q=heads(3), o=heads(3)), dict(o=heads(2)), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")),
              dict(scale=float("inf")), dict(scale=3e38), dict(q=heads(4, None)), dict(o=heads(4, P + 1))):
        assert attend(**k) == dc.DC_EINVAL, k


def test_attend_workspace():
    long = paged(table_pages=4096, table_stride=4096)
    size = L.dc_paged_workspace(byref(long), 4, 1, 0, 0)
    assert size > 0 and size % (2 * 4 * 66 * 4) == 0                             # whole rows of results, base, sum
    assert L.dc_paged_workspace(byref(paged()), 4, 3, 0, 0) == 0                 # a short cache is not split
    assert L.dc_paged_workspace(byref(long), 4, 1, 20, 10) == 0                  # nor a short window
    for ws, n in ((None, size), (P, size - 1), (P + 4, size)):
        assert attend(c=long, s=span(n=1), ws=ws, size=n) == dc.DC_EINVAL and b"workspace" in L.dc_block_last_error()
    for args in ((3, 1, 0, 0), (0, 1, 0, 0), (4, 0, 0, 0), (4, 1, -1, 0), (4, 1, 5, -1), (4, MAX, 0, 0)):
        assert L.dc_paged_workspace(byref(long), *args) == 0
    assert L.dc_paged_workspace(None, 4, 1, 0, 0) == 0


def test_a_call_of_no_tokens_launches_nothing():
    none, c, s = rows(data=None), call(n=0), span(n=0)
    assert residual(c=c, x=none, h=none, r=none, pre=norm(), y=none) == dc.DC_OK
    assert linear(c=c, x=none, out=none) == dc.DC_OK
    assert append(s=s, k=heads(data=None), v=heads(data=None)) == dc.DC_OK
    assert attend(s=s, q=heads(4, None), o=heads(4, None)) == dc.DC_OK
