"""Python binding of the paged cache of include/dc_flow.h: keys and values in
pages of a pool, reached through a table, and the attention over them.

Argument marshalling only, as in carry4.py; for inference, no gradients are
recorded."""
from __future__ import annotations

from ctypes import byref

from .block import _check, _launch, _t
from .carry4 import _INT32, _dtype, _frame, _out, _refuse, _rows, _span
from .carry4 import _pack_rows as _packs
from .flow import DcHeadRows, DcPaged, DcSpan, flib

DC_PAGED_ABI_VERSION = 1
_pack_rows = _packs[2]


def _pool(x, name: str):
    if x.dim() != 4:
        _refuse(f"{name} must have four dimensions, not {x.dim()}")
    sp, st, sh, sd = x.stride()
    if sd != 1:
        _refuse(f"{name}: a head's elements must be consecutive")
    if (sp == 0 and x.shape[0] > 1) or (st == 0 and x.shape[1] > 1) or (sh == 0 and x.shape[2] > 1):
        _refuse(f"{name}: rows that overlap each other's")
    return x.data_ptr(), (sp, st, sh)


class PagedCarry:
    """Keys and values of entries in pages: k_pages, v_pages
    [pages][page_size][heads][head_dim] (float32 or bfloat16, any strides with
    consecutive elements of a head and rows aligned to 16 bytes; page_size a
    power of two, head_dim 64 or 128) and table [batch][table_pages] int32:
    position p of entry b lies in page table[b][p // page_size].  A page number
    outside the pool is a hole: nothing is stored there or seen.  The tensors
    are the caller's and are used in place, the table's values as they are when
    a call runs; positions and lengths stay with the caller too.  attend shares
    out its work by the positions that the table has room for: of a table much
    longer than its entries, pass table[:, :pages] of those in use."""

    def __init__(self, k_pages, v_pages, table):
        torch = _t()
        dt = _dtype(k_pages, "k_pages")
        if v_pages.dtype != k_pages.dtype or v_pages.device != k_pages.device or v_pages.shape != k_pages.shape:
            _refuse("v_pages must have k_pages' type, device and shape")
        (pk, sk), (pv, sv) = _pool(k_pages, "k_pages"), _pool(v_pages, "v_pages")
        pages, page_size, heads, head_dim = k_pages.shape
        if table.dtype != torch.int32 or table.device != k_pages.device or table.dim() != 2 or (table.stride(1) != 1 and table.shape[1] > 1):
            _refuse(f"table must be int32 [batch][table_pages] on {k_pages.device}, with consecutive elements of an entry")
        batch, per = table.shape
        if max(batch, pages, page_size, heads, head_dim, per) > _INT32:
            _refuse("sizes must be below 2^31")
        self.batch, self.heads, self.head_dim, self.page_size = batch, heads, head_dim, page_size
        self.k_pages, self.v_pages, self.table, self.device, self.dtype = k_pages, v_pages, table, k_pages.device, k_pages.dtype
        self.c = DcPaged(DC_PAGED_ABI_VERSION, batch, heads, head_dim, dt, page_size, pages, per, table.data_ptr(), table.stride(0),
                         pk, pv, *sk, *sv)
        self._ref = byref(self.c)
        # (a call of no tokens launches nothing, and checks the pool and the table)
        none = byref(DcHeadRows(None, 0, 0, 0, heads))
        _check(flib().dc_paged_append(self._ref, byref(DcSpan(table.data_ptr(), None, None, batch, 0)), none, none, None))

    def append(self, k, v, pos, lens=None):
        """Store k, v [batch][n][heads][head_dim] at positions pos[b] + i: pos
        int64 [batch], lens int32 [batch] or None.  Positions past the table
        and holes are left out."""
        n = k.shape[1] if k.dim() == 4 else 0
        a = _rows(k, "k", self.device, self.dtype, self.batch, n, self.heads, self.head_dim)
        b = _rows(v, "v", self.device, self.dtype, self.batch, n, self.heads, self.head_dim)
        s = _span(self.device, self.batch, n, pos, lens, None)
        _pack_rows(_frame.rows_, 0, *a, *b)
        _launch(self.device, flib().dc_paged_append, self._ref, s, *_frame.rows[:2])

    def attend(self, q, pos, window: int | None = None, lens=None, sinks: int = 0, causal: bool = True, scale: float | None = None,
               out=None):
        """softmax(scale q k^T) v of q [batch][n][q_heads][head_dim] over the
        cache (which holds the call's own tokens already).  A query at position
        p sees, causal, the positions up to p; else those in [0, pos + len) of
        its entry.  With a window of those the first `sinks` and, causal, the
        ones > p - window; else the ones >= pos - window.  scale: head_dim **
        -0.5 by default.  Rows behind lens are left as they are (zeros where
        out is None).  out may be q itself."""
        torch = _t()
        w = 0 if window is None else window
        if window is not None and not 1 <= window <= _INT32 or not 0 <= sinks <= _INT32:
            _refuse(f"window must be None or in [1, 2^31) and sinks in [0, 2^31), not {window} and {sinks}")
        n = q.shape[1] if q.dim() == 4 else 0
        a = _rows(q, "q", self.device, self.dtype, self.batch, n, None, self.head_dim)
        if out is None:
            out = (torch.empty if lens is None else torch.zeros)(q.shape, dtype=q.dtype, device=self.device)
        o = _out(out, "out", self.device, self.dtype, self.batch, n, a[4], self.head_dim)
        if n and o[0] == a[0] and o[1:4] != a[1:4]:
            _refuse("out: rows that overlap q's")
        s = _span(self.device, self.batch, n, pos, lens, None)
        L = flib()
        size = L.dc_paged_workspace(self._ref, a[4], n, w, sinks)
        # (held until both launches are on the stream: another thread may take freed memory at once)
        ws = torch.empty(size, dtype=torch.uint8, device=self.device) if size else None
        _pack_rows(_frame.rows_, 0, *a, *o)
        _launch(self.device, L.dc_paged_attend, self._ref, s, *_frame.rows[:2], w, sinks, int(causal),
                self.head_dim ** -0.5 if scale is None else scale, ws.data_ptr() if size else None, size)
        return out
