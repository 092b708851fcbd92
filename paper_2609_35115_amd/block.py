"""Python binding of a block's operators of include/dc_flow.h: the norms before
and after a sublayer with its gate and residual, and the matrix product with an
epilogue.

Argument marshalling only, over torch tensors on one GPU; every step runs in
the gfx950 kernels of libdc.so on the caller's current stream, as a torch
operation does (a captured call takes the values of lens at each replay).
Arguments that the C call would misread raise DcError before anything is
launched.  For inference: no gradients are recorded.
"""
from __future__ import annotations

import struct
import threading
from ctypes import byref

from . import carry4
from .carry4 import _INT32, _index, _refuse, _vector
from .flow import DcCall, DcLinearLayer, DcNorm, DcRows, flib
from . import DcError

_KINDS = {"rms": 1, "layer": 2}
_ACTS = {"none": (0, 0), "gelu": (1, 0), "silu": (2, 0), "none_glu": (0, 1), "gelu_glu": (1, 1), "silu_glu": (2, 1)}
_NONE = (0, 0, 0, 0)   # the fields of a row set that is left out


class _Frame(threading.local):
    """A thread's argument structures, filled by one pack a call."""

    def __init__(self):
        self.rows_, self.call_, self.layer_ = bytearray(7 * 32), bytearray(16), bytearray(48)
        self.rows = [byref(DcRows.from_buffer(self.rows_, 32 * i)) for i in range(7)]
        self.call, self.layer = byref(DcCall.from_buffer(self.call_)), byref(DcLinearLayer.from_buffer(self.layer_))


_frame = _Frame()
_pack_rows = {n: struct.Struct("@" + n * "Pqqi4x").pack_into for n in (4, 7)}
_pack_call = struct.Struct("@Pii").pack_into
_pack_layer = struct.Struct("@PPqiiiii4x").pack_into
_device = None   # the current device's index


def _t():
    global _device
    torch = carry4._t()
    if _device is None:
        # (torch's own raw query, as for the stream: a quarter of the time)
        _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return torch


def _check(status: int):
    if status:
        raise DcError(status, flib().dc_block_last_error().decode())


def _launch(device, fn, *args):
    """fn(*args, stream) on the device's current stream."""
    index = device.index
    if index != _device():
        with _t().cuda.device(device):
            return _check(fn(*args, carry4._stream(index)))
    _check(fn(*args, carry4._stream(index)))


def _type(x, name: str) -> int:
    dt = carry4._dtypes.get(x.dtype)
    if dt is None:
        _refuse(f"{name} must be float32 or bfloat16, not {x.dtype}")
    return dt


def _overlap(sb: int, st: int, batch: int, n: int, width: int) -> bool:
    """Whether rows of `width` elements at e sb + i st may share elements."""
    if n == 0:
        return False
    if batch == 1 or n == 1:
        return (sb if n == 1 else st) < width and batch * n > 1
    a, b = ((st, n), (sb, batch)) if st <= sb else ((sb, batch), (st, n))
    return a[0] < width or b[0] < a[0] * a[1]


def _rows(x, name: str, device, shape, out=False):
    """The fields of a row set of x, which has to be of `shape` [batch][n][width]."""
    if x.shape != shape:
        _refuse(f"{name} must be {list(shape)}, not {list(x.shape)}")
    if x.device != device:
        _refuse(f"{name} must be on {device}, not on {x.device}")
    sb, st, sc = x.stride()
    if sc != 1 and shape[2] > 1:
        _refuse(f"{name}: a row's elements must be consecutive")
    if out and _overlap(sb, st, *shape):
        _refuse(f"{name}: rows that overlap each other's")
    dt = carry4._dtypes.get(x.dtype)
    return x.data_ptr(), sb, st, _type(x, name) if dt is None else dt


def _mod(x, name: str, device, shape):
    """The fields of a gate, scale or shift: [width], [batch][width], or three
    dimensions of which the first two may be 1."""
    if x is None:
        return _NONE
    batch, n, width = shape
    own, strides = x.shape, x.stride()
    if x.device != device or not 1 <= len(own) <= 3 or own[-1] != width:
        _refuse(f"{name} must be [{width}], [{batch}][{width}] or [{batch}][{n}][{width}] on {device}, not {list(own)} on {x.device}")
    if strides[-1] != 1 and width > 1:
        _refuse(f"{name}: a row's elements must be consecutive")
    sb = st = 0
    if len(own) > 1 and own[0] != 1:
        sb = strides[0]
        if own[0] != batch:
            _refuse(f"{name} has {own[0]} entries, not {batch}")
    if len(own) > 2 and own[1] != 1:
        st = strides[1]
        if own[1] != n:
            _refuse(f"{name} has {own[1]} tokens, not {n}")
    return x.data_ptr(), sb, st, _type(x, name)


def _shape(x, name: str):
    if not x.is_cuda:
        _refuse(f"{name} must be on a GPU, not {x.device}")
    shape = x.shape
    if len(shape) != 3:
        _refuse(f"{name} must have three dimensions, not {len(shape)}")
    if max(shape) > _INT32 or shape[0] == 0:
        _refuse(f"{name}: sizes must be below 2^31 and the batch at least 1, not {list(shape)}")
    return shape


def _call(device, batch: int, n: int, lens):
    _pack_call(_frame.call_, 0, 0 if lens is None else _index(lens, "lens", device, carry4._torch.int32, batch), batch, n)
    return _frame.call


class Norm:
    """A norm's weights: kind "rms", x / sqrt(mean(x^2) + eps) gain + bias, or
    "layer", the same of x less its mean; gain and bias float32 [width] or None."""

    def __init__(self, kind: str, gain=None, bias=None, eps: float = 1e-6):
        _t()
        if kind not in _KINDS:
            _refuse(f"kind must be one of {sorted(_KINDS)}, not {kind!r}")
        self.kind, self.gain, self.bias, self.eps = kind, gain, bias, eps
        first = gain if gain is not None else bias
        self.device, self.width = (None, None) if first is None else (first.device, first.shape[0] if first.dim() else None)
        self.c = DcNorm(_KINDS[kind], eps, _vector(gain, "gain", self.device, self.width) or None,
                        _vector(bias, "bias", self.device, self.width) or None)
        self._ref = byref(self.c)


def _norm(m, name: str, device, width: int):
    if m is None:
        return None
    if m.width is not None and (m.width != width or m.device != device):
        _refuse(f"{name}: weights must be [{width}] on {device}, not [{m.width}] on {m.device}")
    return m._ref


def norm_residual(x, h=None, *, post=None, gate=None, x_scale: float = 1.0, pre=None, scale=None, shift=None, lens=None, out=None):
    """(r, y) of the residual stream x and a sublayer's result h [batch][n][width]:

        r = x_scale x + gate post(h),    y = pre(r) (1 + scale) + shift

    in one pass (r enters y before it is rounded).  post, pre: Norm or None (the
    identity); gate, scale, shift: None, [width], [batch][width] or
    [batch][n][width].  Each tensor float32 or bfloat16; r has x's type, y has
    h's.  h None: r = x_scale x, and only y is computed (in x's type, or in
    out's).  y is None where pre, scale and shift are.  Widths to 16384.  lens
    int32 [batch] or None: rows behind an entry's lens are left as they are
    (zeros where out is None).  out: the two results' tensors, either of which
    may be None (that result is not stored); they may be x and h (r in x, y in h)
    and share no memory with another argument otherwise."""
    torch = _t()
    shape = _shape(x, "x")
    B, n, W = shape
    device, dx = x.device, x.dtype
    dy = dx if h is None else h.dtype
    if h is None and (post is not None or gate is not None):
        _refuse("post and gate go with h")
    fx, fh = _rows(x, "x", device, shape), _NONE if h is None else _rows(h, "h", device, shape)
    more = pre is not None or scale is not None or shift is not None
    if out is None:
        new = torch.empty if lens is None else torch.zeros
        r = new(shape, dtype=dx, device=device) if h is not None else None
        y = new(shape, dtype=dy, device=device) if more else None
    else:
        r, y = out
    if r is None and y is None:
        _refuse("nothing to compute: neither r nor y")
    if y is None and more:
        _refuse("pre, scale and shift go with y")
    fr = fy = _NONE
    # (an address with the same strides and type is the same rows)
    if r is not None:
        fr = _rows(r, "out[0]", device, shape, True)
        if r.dtype != dx:
            _refuse(f"out[0] must be {dx} as x is, not {r.dtype}")
        if n and (fr[0] == fx[0] and fr != fx or fr[0] == fh[0] and fr != fh):
            _refuse("out[0]: rows that overlap another argument's")
    if y is not None:
        fy = _rows(y, "out[1]", device, shape, True)
        if h is not None and y.dtype != dy:
            _refuse(f"out[1] must be {dy} as h is, not {y.dtype}")
        if n and (fy[0] == fr[0] or fy[0] == fh[0] and fy != fh or fy[0] == fx[0] and fy != fx):
            _refuse("out[1]: rows that overlap another argument's")
    f = _frame.rows
    _pack_rows[7](_frame.rows_, 0, *fx, *fh, *_mod(gate, "gate", device, shape), *fr, *_mod(scale, "scale", device, shape),
                  *_mod(shift, "shift", device, shape), *fy)
    _launch(device, flib().dc_norm_residual, _call(device, B, n, lens), W, f[0], x_scale, None if h is None else f[1],
            None if post is None else _norm(post, "post", device, W), None if gate is None else f[2], None if r is None else f[3],
            None if pre is None else _norm(pre, "pre", device, W), None if scale is None else f[4], None if shift is None else f[5],
            None if y is None else f[6])
    return r, y


def linear(x, weight, bias=None, act: str = "none", gate=None, residual=None, residual_scale: float = 1.0, lens=None, out=None,
           out_dtype=None):
    """residual_scale residual + gate act(x weight^T + bias) of x [batch][n][n_in],
    accumulated in float32 and rounded once.  weight: x's type (float32 or
    bfloat16), [n_out][n_in], or [2 n_out][n_in] for the acts "..._glu": the
    first half is activated, the other half multiplied with the result.  act:
    "none", "gelu" (tanh form), "silu", "none_glu", "gelu_glu", "silu_glu".  bias
    float32, one value a row of the weight.  gate: None, [n_out],
    [batch][n_out] or [batch][n][n_out]; residual [batch][n][n_out]; both
    float32 or bfloat16.  lens int32 [batch] or None: rows behind an entry's
    lens are left as they are (zeros where out is None).  out (of either type;
    where it is None, a new one of x's type or out_dtype) may be residual itself,
    and shares no memory with another argument otherwise."""
    torch = _t()
    shape = _shape(x, "x")
    B, n, K = shape
    device, dtype = x.device, x.dtype
    code = _ACTS.get(act)
    if code is None:
        _refuse(f"act must be one of {sorted(_ACTS)}, not {act!r}")
    if weight.dim() != 2 or weight.shape[1] != K or weight.dtype != dtype or weight.device != device:
        _refuse(f"weight must be {dtype} [n_out][{K}] on {device}, not {weight.dtype} {list(weight.shape)} on {weight.device}")
    R = weight.shape[0]
    if code[1] and R % 2:
        _refuse(f"weight needs an even number of rows for {act}, not {R}")
    N = R // 2 if code[1] else R
    ws, wc = weight.stride()
    if (wc != 1 and K > 1) or N > _INT32:
        _refuse("weight: a row's elements must be consecutive")
    if R == 1:
        ws = K
    result = torch.Size((B, n, N))
    fx, fg = _rows(x, "x", device, shape), _mod(gate, "gate", device, result)
    fr = _NONE if residual is None else _rows(residual, "residual", device, result)
    if out is None:
        out = (torch.empty if lens is None else torch.zeros)(result, dtype=out_dtype or dtype, device=device)
    elif out_dtype is not None and out.dtype != out_dtype:
        _refuse(f"out must be {out_dtype}, not {out.dtype}")
    fo = _rows(out, "out", device, result, True)
    pw = weight.data_ptr()
    # (an address with the same strides and type is the same rows)
    if n and (fo[0] == fx[0] or fo[0] == pw or fo[0] == fr[0] and fo != fr):
        _refuse("out: rows that overlap another argument's")
    _pack_layer(_frame.layer_, 0, pw, 0 if bias is None else _vector(bias, "bias", device, R), ws, K, N, fx[3], *code)
    _pack_rows[4](_frame.rows_, 0, *fx, *fg, *fr, *fo)
    f, L = _frame.rows, flib()
    size = L.dc_linear_workspace(_frame.layer, B, n)
    # (held until both launches are on the stream: another thread may take freed memory at once)
    w = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    _launch(device, L.dc_linear, _call(device, B, n, lens), _frame.layer, f[0], None if gate is None else f[1],
            None if residual is None else f[2], residual_scale, f[3], w.data_ptr() if size else None, size)
    return out
