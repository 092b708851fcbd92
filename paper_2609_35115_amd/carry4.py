"""Python binding of the attention operators of include/dc_flow.h: per-head
norms with the position rotation, a carry of keys and values held in 4 bits,
and the attention over it.

Argument marshalling only, over torch tensors on one GPU; every step runs in
the gfx950 kernels of libdc.so on the caller's current stream, as a torch
operation does (a captured call takes the values of pos, lens and sinks at
each replay).  Arguments that the C call would misread raise DcError before
anything is launched.  For inference: no gradients are recorded.
"""
from __future__ import annotations

import struct
import threading
from ctypes import byref

from . import DC_BF16, DC_EINVAL, DC_F32, DcError
from .flow import DcCarry4, DcHeadRows, DcQkNorm, DcSpan, flib

DC_CARRY4_ABI_VERSION = 1
_INT32 = 2 ** 31 - 1   # ctypes cuts integers to their field without a word

_torch = None
_dtypes = {}
_stream = None   # device index -> the current stream's handle


def _t():
    global _torch, _stream
    if _torch is None:
        import torch
        _dtypes.update({torch.float32: DC_F32, torch.bfloat16: DC_BF16})
        # torch's own raw query: building a Stream object takes 2.8 us, a third of a small call
        _stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda index: torch.cuda.current_stream(index).cuda_stream)
        _torch = torch
    return _torch


class _Frame(threading.local):
    """A thread's argument structures, filled by one pack a kind: building them
    anew takes 2 us of a call of four row sets."""

    def __init__(self):
        self.rows_, self.span_, self.norm_ = bytearray(4 * 40), bytearray(32), bytearray(40)
        self.rows = [byref(DcHeadRows.from_buffer(self.rows_, 40 * i)) for i in range(4)]
        self.span, self.norm = byref(DcSpan.from_buffer(self.span_)), byref(DcQkNorm.from_buffer(self.norm_))


_frame = _Frame()
_pack_rows = {n: struct.Struct("@" + n * "Pqqqi4x").pack_into for n in (2, 4)}
_pack_span = struct.Struct("@PPPii").pack_into
_pack_norm = struct.Struct("@PPPiif4x").pack_into


def _refuse(why: str):
    raise DcError(DC_EINVAL, why)


def _check(status: int):
    if status:
        raise DcError(status, flib().dc_carry4_last_error().decode())


def _rows(x, name: str, device, dtype, batch: int, n: int, heads, head_dim: int):
    """The fields of a row set of x [batch][n][heads][head_dim], in place."""
    if x.dtype != dtype or x.device != device:
        _refuse(f"{name} must be {dtype} on {device}, not {x.dtype} on {x.device}")
    shape = x.shape
    if len(shape) != 4:
        _refuse(f"{name} must have four dimensions, not {len(shape)}")
    b, t, h, d = shape
    if b != batch or t != n or d != head_dim or (heads and h != heads):
        _refuse(f"{name} must be [{batch}][{n}][{heads or 'heads'}][{head_dim}], not {list(shape)}")
    if t > _INT32 or h > _INT32:
        _refuse(f"{name}: tokens and heads must be below 2^31, not {t} and {h}")
    sb, st, sh, sd = x.stride()
    if sd != 1:
        _refuse(f"{name}: a head's elements must be consecutive")
    return x.data_ptr(), sb, st, sh, h


def _out(x, name: str, device, dtype, batch: int, n: int, heads, head_dim: int, *others):
    """_rows of a result, whose rows have places of their own: none shared with
    each other, nor with the row sets `others` (by their first element)."""
    r = _rows(x, name, device, dtype, batch, n, heads, head_dim)
    if (r[1] == 0 and batch > 1) or (r[2] == 0 and n > 1) or (r[3] == 0 and r[4] > 1) or (n and r[0] in others):
        _refuse(f"{name}: rows that overlap each other's, or those of another argument")
    return r


def _index(x, name: str, device, dtype, batch: int) -> int:
    """Address of a device array [batch] (None: NULL)."""
    if x is None:
        return 0
    if x.dtype != dtype or x.device != device or x.dim() != 1 or x.shape[0] != batch or not x.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor [{batch}] on {device}")
    return x.data_ptr()


def _span(device, batch: int, n: int, pos, lens, sinks):
    torch = _torch
    if pos is None:
        _refuse("pos is None")
    _pack_span(_frame.span_, 0, _index(pos, "pos", device, torch.int64, batch), _index(lens, "lens", device, torch.int32, batch),
               _index(sinks, "sinks", device, torch.int32, batch), batch, n)
    return _frame.span


def _vector(x, name: str, device, size) -> int:
    """Address of a float32 vector (None: NULL)."""
    if x is None:
        return 0
    if x.dtype != _torch.float32 or x.device != device or x.dim() != 1 or not x.is_contiguous() or (size and x.shape[0] != size):
        _refuse(f"{name} must be a contiguous float32 tensor{f' [{size}]' if size else ''} on {device}")
    return x.data_ptr()


def _norm(device, head_dim: int, freqs, q_gain, k_gain, eps: float, interleaved: bool):
    a, b = _vector(q_gain, "q_gain", device, head_dim), _vector(k_gain, "k_gain", device, head_dim)
    f, nf = _vector(freqs, "freqs", device, None), 0 if freqs is None else freqs.shape[0]
    try:
        _pack_norm(_frame.norm_, 0, a, b, f, nf, int(interleaved), eps)
    except (struct.error, OverflowError):
        _refuse(f"eps or the number of frequencies does not fit its field: {eps}, {nf}")
    return _frame.norm


def _dtype(x, name: str) -> int:
    _t()
    dt = _dtypes.get(x.dtype)
    if dt is None:
        _refuse(f"{name} must be float32 or bfloat16, not {x.dtype}")
    if not x.is_cuda:
        _refuse(f"{name} must be on a GPU, not {x.device}")
    if x.dim() != 4:
        _refuse(f"{name} must have four dimensions, not {x.dim()}")
    return dt


def _launch(device, fn, *args):
    """fn(*args, stream) on the device's current stream."""
    if device.index != _torch.cuda.current_device():
        with _torch.cuda.device(device):
            return _check(fn(*args, _stream(device.index)))
    _check(fn(*args, _stream(device.index)))


def qk_norm_rope(q, k, pos, freqs, q_gain=None, k_gain=None, eps: float = 1e-6, interleaved: bool = False, lens=None,
                 out=None):
    """(q', k') of q [batch][n][q_heads][head_dim], k [batch][n][k_heads][head_dim]
    (float32 or bfloat16, any strides with consecutive elements of a head):
    RMS norm per head with the gains [head_dim], then the rotation by
    (pos[b] + i) * freqs [n_freqs] of the first 2 n_freqs dimensions (freqs
    None: no rotation).  pos int64 [batch], lens int32 [batch] or None.  out:
    the two results' tensors, which may be q and k themselves (in that order)
    and share no memory with another argument otherwise; rows behind
    lens are left as they are (zeros where out is None)."""
    dt = _dtype(q, "q")
    device, dtype = q.device, q.dtype
    B, n, Hq, D = q.shape
    a, b = _rows(q, "q", device, dtype, B, n, None, D), _rows(k, "k", device, dtype, B, n, None, D)
    if out is None:
        new = _torch.empty if lens is None else _torch.zeros
        out = (new(q.shape, dtype=dtype, device=device), new(k.shape, dtype=dtype, device=device))
    qo, ko = out
    c = _out(qo, "out[0]", device, dtype, B, n, Hq, D, b[0])
    d = _out(ko, "out[1]", device, dtype, B, n, b[4], D, a[0], c[0])
    m, s = _norm(device, D, freqs, q_gain, k_gain, eps, interleaved), _span(device, B, n, pos, lens, None)
    _pack_rows[4](_frame.rows_, 0, *a, *b, *c, *d)
    _launch(device, flib().dc_qk_norm_rope, m, s, D, dt, *_frame.rows)
    return qo, ko


class Carry4:
    """Keys and values of `batch` entries in 4 bits: their first `sinks` tokens,
    and a ring of the `ring` tokens after them.  `memory` is a uint8 tensor;
    positions and lengths stay with the caller."""

    def __init__(self, batch: int, heads: int, head_dim: int, sinks: int, ring: int, device=None):
        torch = _t()
        if not all(0 <= x <= _INT32 for x in (batch, heads, head_dim, sinks, ring)):
            _refuse("batch, heads, head_dim, sinks and ring must be in [0, 2^31)")
        self.batch, self.heads, self.head_dim, self.sinks, self.ring = batch, heads, head_dim, sinks, ring
        self.c = DcCarry4(DC_CARRY4_ABI_VERSION, batch, heads, head_dim, sinks, ring, None)
        size = flib().dc_carry4_bytes(byref(self.c))
        if size == 0:
            raise DcError(DC_EINVAL, flib().dc_carry4_last_error().decode())
        self.memory = torch.empty(size, dtype=torch.uint8, device=torch.device("cuda" if device is None else device))
        self.device = self.memory.device
        self.c.data = self.memory.data_ptr()
        self._ref = byref(self.c)

    @property
    def bytes(self) -> int:
        return self.memory.numel()

    def _kv(self, k, v):
        """(dtype, n, fields of k, of v)."""
        dt, dtype = _dtype(k, "k"), k.dtype
        n = k.shape[1]
        return (dt, n, _rows(k, "k", self.device, dtype, self.batch, n, self.heads, self.head_dim),
                _rows(v, "v", self.device, dtype, self.batch, n, self.heads, self.head_dim))

    def append(self, k, v, pos, lens=None, sinks=None):
        """Store k, v [batch][n][heads][head_dim] at positions pos[b] + i."""
        dt, n, a, b = self._kv(k, v)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        _pack_rows[2](_frame.rows_, 0, *a, *b)
        _launch(self.device, flib().dc_carry4_append, self._ref, None, s, dt, None, *_frame.rows[:2], None)

    def append_rotated(self, q, k, v, pos, freqs, q_gain=None, k_gain=None, eps: float = 1e-6, interleaved: bool = False,
                       lens=None, sinks=None, out=None):
        """qk_norm_rope of q and k and the store of the keys and v in one pass;
        returns the queries."""
        dt, n, a, b = self._kv(k, v)
        r = _rows(q, "q", self.device, k.dtype, self.batch, n, None, self.head_dim)
        if out is None:
            out = (_torch.empty if lens is None else _torch.zeros)(q.shape, dtype=q.dtype, device=self.device)
        o = _out(out, "out", self.device, k.dtype, self.batch, n, r[4], self.head_dim, a[0], b[0])
        m = _norm(self.device, self.head_dim, freqs, q_gain, k_gain, eps, interleaved)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        _pack_rows[4](_frame.rows_, 0, *r, *a, *b, *o)
        _launch(self.device, flib().dc_carry4_append, self._ref, m, s, dt, *_frame.rows)
        return out

    def attend(self, q, pos, window: int, lens=None, sinks=None, causal: bool = True, scale: float | None = None, out=None):
        """softmax(scale q k^T) v of q [batch][n][q_heads][head_dim] over the
        carry (which holds the call's own tokens already): the first tokens
        and, causal, the positions in (p - window, p] of a query at p; else
        those in [pos - window, pos + len) for all of an entry's queries.
        Only as far as the ring still holds them after the call's last token:
        it needs window + n slots (causal: one less) for early queries to see
        their whole window; calls of up to ring + sinks are taken, for entries
        that begin among their first tokens, and past those an early query sees
        fewer keys, or none (0).  scale: head_dim ** -0.5 by default.  out may
        be q itself."""
        dt, dtype = _dtype(q, "q"), q.dtype
        if not 0 <= window <= _INT32:
            _refuse(f"window must be in [0, 2^31), not {window}")
        n = q.shape[1]
        a = _rows(q, "q", self.device, dtype, self.batch, n, None, self.head_dim)
        if out is None:
            out = (_torch.empty if lens is None else _torch.zeros)(q.shape, dtype=dtype, device=self.device)
        o = _out(out, "out", self.device, dtype, self.batch, n, a[4], self.head_dim)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        L = flib()
        size = L.dc_carry4_workspace(self._ref, a[4], n, window)
        # (held until both launches are on the stream: another thread may take freed memory at once)
        ws = _torch.empty(size, dtype=_torch.uint8, device=self.device) if size else None
        _pack_rows[2](_frame.rows_, 0, *a, *o)
        _launch(self.device, L.dc_carry4_attend, self._ref, s, dt, *_frame.rows[:2], window, int(causal),
                self.head_dim ** -0.5 if scale is None else scale, ws.data_ptr() if size else None, size)
        return out

    def read(self, pos, n: int, lens=None, sinks=None, dtype=None):
        """(k, v) [batch][n][heads][head_dim]: the values held for positions
        pos[b] + i (float32 or bfloat16, exact in both)."""
        new = _t().empty if lens is None else _torch.zeros
        k, v = new((2, self.batch, n, self.heads, self.head_dim), dtype=dtype or _torch.float32, device=self.device)
        dt, n, a, b = self._kv(k, v)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        _pack_rows[2](_frame.rows_, 0, *a, *b)
        _launch(self.device, flib().dc_carry4_read, self._ref, s, dt, *_frame.rows[:2])
        return k, v
