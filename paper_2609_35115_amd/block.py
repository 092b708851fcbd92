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
from .carry4 import _INT32, _index, _refuse, _t, _vector
from .flow import DcCall, DcLinearLayer, DcNorm, DcRows, flib
from . import DcError

_KINDS = {"rms": 1, "layer": 2}
_ACTS = {"none": (0, 0), "gelu": (1, 0), "silu": (2, 0), "none_glu": (0, 1), "gelu_glu": (1, 1), "silu_glu": (2, 1)}


class _Frame(threading.local):
    """A thread's argument structures, filled by one pack a kind."""

    def __init__(self):
        self.rows_, self.call_, self.layer_ = bytearray(7 * 32), bytearray(16), bytearray(48)
        self.rows = [byref(DcRows.from_buffer(self.rows_, 32 * i)) for i in range(7)]
        self.call, self.layer = byref(DcCall.from_buffer(self.call_)), byref(DcLinearLayer.from_buffer(self.layer_))


_frame = _Frame()
_pack_rows = struct.Struct("@Pqqi4x").pack_into
_pack_call = struct.Struct("@Pii").pack_into
_pack_layer = struct.Struct("@PPqiiiii4x").pack_into


def _check(status: int):
    if status:
        raise DcError(status, flib().dc_block_last_error().decode())


def _launch(device, fn, *args):
    """fn(*args, stream) on the device's current stream."""
    torch = _t()
    if device.index != torch.cuda.current_device():
        with torch.cuda.device(device):
            return _check(fn(*args, carry4._stream(device.index)))
    _check(fn(*args, carry4._stream(device.index)))


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


def _rows(at: int, x, name: str, device, batch: int, n: int, width: int, out=False):
    """Fills row set `at` with x [batch][n][width]; its first element's address."""
    if x.dim() != 3 or x.shape[0] != batch or x.shape[1] != n or x.shape[2] != width:
        _refuse(f"{name} must be [{batch}][{n}][{width}], not {list(x.shape)}")
    if x.device != device:
        _refuse(f"{name} must be on {device}, not on {x.device}")
    sb, st, sc = x.stride()
    if sc != 1 and width > 1:
        _refuse(f"{name}: a row's elements must be consecutive")
    if out and _overlap(sb, st, batch, n, width):
        _refuse(f"{name}: rows that overlap each other's")
    p = x.data_ptr()
    _pack_rows(_frame.rows_, 32 * at, p, sb, st, _type(x, name))
    return p


def _mod(at: int, x, name: str, device, batch: int, n: int, width: int):
    """Row set `at` of a gate, scale or shift: [width], [batch][width], or three
    dimensions of which the first two may be 1.  None: NULL."""
    if x is None:
        return None
    shape, strides = x.shape, x.stride()
    if x.device != device or not 1 <= len(shape) <= 3 or shape[-1] != width:
        _refuse(f"{name} must be [{width}], [{batch}][{width}] or [{batch}][{n}][{width}] on {device}, not {list(shape)} on {x.device}")
    if strides[-1] != 1 and width > 1:
        _refuse(f"{name}: a row's elements must be consecutive")
    sb = st = 0
    if len(shape) > 1 and shape[0] != 1:
        sb = strides[0]
        if shape[0] != batch:
            _refuse(f"{name} has {shape[0]} entries, not {batch}")
    if len(shape) > 2 and shape[1] != 1:
        st = strides[1]
        if shape[1] != n:
            _refuse(f"{name} has {shape[1]} tokens, not {n}")
    _pack_rows(_frame.rows_, 32 * at, x.data_ptr(), sb, st, _type(x, name))
    return _frame.rows[at]


def _shape(x, name: str):
    if not x.is_cuda:
        _refuse(f"{name} must be on a GPU, not {x.device}")
    if x.dim() != 3:
        _refuse(f"{name} must have three dimensions, not {x.dim()}")
    b, n, w = x.shape
    if max(b, n, w) > _INT32 or b == 0:
        _refuse(f"{name}: sizes must be below 2^31 and the batch at least 1, not {list(x.shape)}")
    return b, n, w


def _call(device, batch: int, n: int, lens):
    import torch
    _pack_call(_frame.call_, 0, _index(lens, "lens", device, torch.int32, batch), batch, n)
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
    h's.  h None: r = x_scale x, and only y is computed.  y is None where pre,
    scale and shift are.  lens int32 [batch] or None: rows behind an entry's
    lens are left as they are (zeros where out is None).  out: the two results'
    tensors, either of which may be None (that result is not stored); they may
    be x and h (r in x, y in h) and share no memory with another argument
    otherwise."""
    torch = _t()
    B, n, W = _shape(x, "x")
    device = x.device
    px = _rows(0, x, "x", device, B, n, W)
    if h is None and (post is not None or gate is not None):
        _refuse("post and gate go with h")
    ph = _rows(1, h, "h", device, B, n, W) if h is not None else None
    more = pre is not None or scale is not None or shift is not None
    if out is None:
        new = torch.empty if lens is None else torch.zeros
        r = new(x.shape, dtype=x.dtype, device=device) if h is not None else None
        y = new(x.shape, dtype=x.dtype if h is None else h.dtype, device=device) if more else None
    else:
        r, y = out
    if r is None and y is None:
        _refuse("nothing to compute: neither r nor y")
    if y is None and more:
        _refuse("pre, scale and shift go with y")
    pr = py = None
    if r is not None:
        pr = _rows(3, r, "out[0]", device, B, n, W, True)
        if r.dtype != x.dtype:
            _refuse(f"out[0] must be {x.dtype} as x is, not {r.dtype}")
        if n and W and pr == px and r.stride() != x.stride() or n and W and pr == ph and (r.stride() != h.stride() or r.dtype != h.dtype):
            _refuse("out[0]: rows that overlap another argument's")
    if y is not None:
        py = _rows(6, y, "out[1]", device, B, n, W, True)
        if h is not None and y.dtype != h.dtype:
            _refuse(f"out[1] must be {h.dtype} as h is, not {y.dtype}")
        if n and W and (py == pr or py == ph and y.stride() != h.stride() or py == px and (y.stride() != x.stride() or y.dtype != x.dtype)):
            _refuse("out[1]: rows that overlap another argument's")
    f = _frame.rows
    try:
        _launch(device, flib().dc_norm_residual, _call(device, B, n, lens), W, f[0], x_scale, f[1] if h is not None else None,
                _norm(post, "post", device, W), _mod(2, gate, "gate", device, B, n, W), f[3] if r is not None else None,
                _norm(pre, "pre", device, W), _mod(4, scale, "scale", device, B, n, W), _mod(5, shift, "shift", device, B, n, W),
                f[6] if y is not None else None)
    except OverflowError:
        _refuse(f"x_scale does not fit a float: {x_scale}")
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
    lens are left as they are (zeros where out is None).  out (x's type, or
    out_dtype) may be residual itself, and shares no memory with another
    argument otherwise."""
    torch = _t()
    B, n, K = _shape(x, "x")
    device, dtype = x.device, x.dtype
    if act not in _ACTS:
        _refuse(f"act must be one of {sorted(_ACTS)}, not {act!r}")
    a, glu = _ACTS[act]
    if weight.dim() != 2 or weight.shape[1] != K or weight.dtype != dtype or weight.device != device:
        _refuse(f"weight must be {dtype} [n_out][{K}] on {device}, not {weight.dtype} {list(weight.shape)} on {weight.device}")
    R = weight.shape[0]
    if glu and R % 2:
        _refuse(f"weight needs an even number of rows for {act}, not {R}")
    N = R // 2 if glu else R
    ws, wc = weight.stride()
    if (wc != 1 and K > 1) or N > _INT32:
        _refuse("weight: a row's elements must be consecutive")
    if R == 1:
        ws = K
    px = _rows(0, x, "x", device, B, n, K)
    pb = _vector(bias, "bias", device, R)
    pr = _rows(2, residual, "residual", device, B, n, N) if residual is not None else None
    if out is None:
        out = (torch.empty if lens is None else torch.zeros)((B, n, N), dtype=out_dtype or dtype, device=device)
    elif out_dtype is not None and out.dtype != out_dtype:
        _refuse(f"out must be {out_dtype}, not {out.dtype}")
    po = _rows(3, out, "out", device, B, n, N, True)
    if n and (po == px or po == weight.data_ptr() or po == pr and (out.stride() != residual.stride() or out.dtype != residual.dtype)):
        _refuse("out: rows that overlap another argument's")
    g = _mod(1, gate, "gate", device, B, n, N)
    _pack_layer(_frame.layer_, 0, weight.data_ptr(), pb, ws, K, N, _type(weight, "weight"), a, glu)
    f, L = _frame.rows, flib()
    size = L.dc_linear_workspace(_frame.layer, B, n)
    # (held until both launches are on the stream: another thread may take freed memory at once)
    w = torch.empty(size, dtype=torch.uint8, device=device) if size else None
    try:
        _launch(device, L.dc_linear, _call(device, B, n, lens), _frame.layer, f[0], g, f[2] if residual is not None else None,
                residual_scale, f[3], w.data_ptr() if size else None, size)
    except OverflowError:
        _refuse(f"residual_scale does not fit a float: {residual_scale}")
    return out
