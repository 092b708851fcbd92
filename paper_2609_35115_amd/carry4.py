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

from ctypes import byref

from . import DC_BF16, DC_EINVAL, DC_F32, DcError
from .flow import DcCarry4, DcHeadRows, DcQkNorm, DcSpan, flib

DC_CARRY4_ABI_VERSION = 1

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


def _refuse(why: str):
    raise DcError(DC_EINVAL, why)


def _check(status: int):
    if status:
        raise DcError(status, flib().dc_carry4_last_error().decode())


def _rows(x, name: str, device, dtype, batch: int, n: int, heads, head_dim: int) -> DcHeadRows:
    """A row set of x [batch][n][heads][head_dim], in place."""
    if x.dtype != dtype or x.device != device:
        _refuse(f"{name} must be {dtype} on {device}, not {x.dtype} on {x.device}")
    shape = x.shape
    if len(shape) != 4 or shape[0] != batch or shape[1] != n or shape[3] != head_dim or (heads and shape[2] != heads):
        _refuse(f"{name} must be [{batch}][{n}][{heads or 'heads'}][{head_dim}], not {list(shape)}")
    sb, st, sh, sd = x.stride()
    if sd != 1:
        _refuse(f"{name}: a head's elements must be consecutive")
    return DcHeadRows(x.data_ptr(), sb, st, sh, shape[2])


def _index(x, name: str, device, dtype, batch: int):
    """Address of a device array [batch] (None: NULL)."""
    if x is None:
        return None
    if x.dtype != dtype or x.device != device or x.dim() != 1 or x.shape[0] != batch or not x.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor [{batch}] on {device}")
    return x.data_ptr()


def _span(device, batch: int, n: int, pos, lens, sinks) -> DcSpan:
    torch = _torch
    if pos is None:
        _refuse("pos is None")
    return DcSpan(_index(pos, "pos", device, torch.int64, batch), _index(lens, "lens", device, torch.int32, batch),
                  _index(sinks, "sinks", device, torch.int32, batch), batch, n)


def _norm(device, head_dim: int, freqs, q_gain, k_gain, eps: float, interleaved: bool) -> DcQkNorm:
    torch = _torch
    ptr = []
    for x, name, size in ((q_gain, "q_gain", head_dim), (k_gain, "k_gain", head_dim), (freqs, "freqs", None)):
        if x is None:
            ptr.append(None)
            continue
        if x.dtype != torch.float32 or x.device != device or x.dim() != 1 or not x.is_contiguous() or (
                size and x.shape[0] != size):
            _refuse(f"{name} must be a contiguous float32 tensor{f' [{size}]' if size else ''} on {device}")
        ptr.append(x.data_ptr())
    return DcQkNorm(ptr[0], ptr[1], ptr[2], 0 if freqs is None else freqs.shape[0], int(interleaved), eps)


def _dtype(x, name: str) -> int:
    _t()
    if x.dtype not in _dtypes:
        _refuse(f"{name} must be float32 or bfloat16, not {x.dtype}")
    if x.device.type != "cuda":
        _refuse(f"{name} must be on a GPU, not {x.device}")
    if x.dim() != 4:
        _refuse(f"{name} must have four dimensions, not {x.dim()}")
    return _dtypes[x.dtype]


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
    the two results' tensors, which may be q and k themselves; rows behind
    lens are left as they are (zeros where out is None)."""
    dt = _dtype(q, "q")
    torch, device = _torch, q.device
    B, n, Hq, D = q.shape
    a, b = _rows(q, "q", device, q.dtype, B, n, None, D), _rows(k, "k", device, q.dtype, B, n, None, D)
    if out is None:
        new = torch.empty if lens is None else torch.zeros
        out = (new(q.shape, dtype=q.dtype, device=device), new(k.shape, dtype=q.dtype, device=device))
    c, d = _rows(out[0], "out[0]", device, q.dtype, B, n, Hq, D), _rows(out[1], "out[1]", device, q.dtype, B, n, k.shape[2], D)
    m = _norm(device, D, freqs, q_gain, k_gain, eps, interleaved)
    s = _span(device, B, n, pos, lens, None)
    _launch(device, flib().dc_qk_norm_rope, byref(m), byref(s), D, dt, byref(a), byref(b), byref(c), byref(d))
    return tuple(out)


class Carry4:
    """Keys and values of `batch` entries in 4 bits: their first `sinks` tokens,
    and a ring of the `ring` tokens after them.  `memory` is a uint8 tensor;
    positions and lengths stay with the caller."""

    def __init__(self, batch: int, heads: int, head_dim: int, sinks: int, ring: int, device=None):
        torch = _t()
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

    def _kv(self, k, v, what=("k", "v")):
        dt = _dtype(k, what[0])
        n = k.shape[1]
        return dt, n, *(_rows(x, w, self.device, k.dtype, self.batch, n, self.heads, self.head_dim)
                        for x, w in zip((k, v), what))

    def append(self, k, v, pos, lens=None, sinks=None):
        """Store k, v [batch][n][heads][head_dim] at positions pos[b] + i."""
        dt, n, a, b = self._kv(k, v)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        _launch(self.device, flib().dc_carry4_append, self._ref, None, byref(s), dt, None, byref(a), byref(b), None)

    def append_rotated(self, q, k, v, pos, freqs, q_gain=None, k_gain=None, eps: float = 1e-6, interleaved: bool = False,
                       lens=None, sinks=None, out=None):
        """qk_norm_rope of q and k and the store of the keys and v in one pass;
        returns the queries."""
        dt, n, a, b = self._kv(k, v)
        torch = _torch
        r = _rows(q, "q", self.device, k.dtype, self.batch, n, None, self.head_dim)
        if out is None:
            out = (torch.empty if lens is None else torch.zeros)(q.shape, dtype=q.dtype, device=self.device)
        o = _rows(out, "out", self.device, k.dtype, self.batch, n, q.shape[2], self.head_dim)
        m = _norm(self.device, self.head_dim, freqs, q_gain, k_gain, eps, interleaved)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        _launch(self.device, flib().dc_carry4_append, self._ref, byref(m), byref(s), dt, byref(r), byref(a), byref(b), byref(o))
        return out

    def attend(self, q, pos, window: int, lens=None, sinks=None, causal: bool = True, scale: float | None = None, out=None):
        """softmax(scale q k^T) v of q [batch][n][q_heads][head_dim] over the
        carry (which holds the call's own tokens already): the first tokens
        and, causal, the positions in (p - window, p] of a query at p; else
        those in [pos - window, pos + len) for all of an entry's queries.
        scale: head_dim ** -0.5 by default.  out may be q itself."""
        dt = _dtype(q, "q")
        torch = _torch
        B, n, Hq, _ = q.shape
        a = _rows(q, "q", self.device, q.dtype, self.batch, n, None, self.head_dim)
        if out is None:
            out = (torch.empty if lens is None else torch.zeros)(q.shape, dtype=q.dtype, device=self.device)
        o = _rows(out, "out", self.device, q.dtype, self.batch, n, Hq, self.head_dim)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        L = flib()
        size = L.dc_carry4_workspace(self._ref, Hq, n, window)
        ws = torch.empty(size, dtype=torch.uint8, device=self.device) if size else None
        _launch(self.device, L.dc_carry4_attend, self._ref, byref(s), dt, byref(a), byref(o), window, int(causal),
                self.head_dim ** -0.5 if scale is None else scale, ws.data_ptr() if size else None, size)
        return out

    def read(self, pos, n: int, lens=None, sinks=None, dtype=None):
        """(k, v) [batch][n][heads][head_dim]: the values held for positions
        pos[b] + i (float32 or bfloat16, exact in both)."""
        torch = _t()
        new = torch.empty if lens is None else torch.zeros
        k, v = (new((self.batch, n, self.heads, self.head_dim), dtype=dtype or torch.float32, device=self.device) for _ in "kv")
        dt, n, a, b = self._kv(k, v)
        s = _span(self.device, self.batch, n, pos, lens, sinks)
        _launch(self.device, flib().dc_carry4_read, self._ref, byref(s), dt, byref(a), byref(b))
        return k, v
