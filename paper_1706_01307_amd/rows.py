"""Operators on feature rows, as used between sparse convolutions.

    y, mean, rstd = layer_norm_forward(x, gamma, beta)
    r = route_forward(logits, k)                               # r.rows, r.offsets, r.pos, ...
    h = grouped_forward(y, w1, r.offsets, rows=r.rows, bias=b1, relu=True)
    z = grouped_forward(h, w2, r.offsets, bias=b2)
    u = combine_forward(z, r.pos, r.weights)
    out = dropout_forward(u, 0.1, seed, offset=step, residual=x)

Argument marshalling only (the C ABI is include/spconv_rows.h).  Tensors are on
torch's current device; inputs that are not contiguous are copied.  Everything,
copies included, runs on torch's current stream or on `stream`; tensors made on
another stream are the caller's to order, as for torch's own operators.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools

from . import _lib
from ._lib import ROUTE_MAX_EXPERTS, ROUTE_MAX_SLOTS

__all__ = ["Routing", "layer_norm_forward", "layer_norm_backward", "dropout_forward",
           "dropout_backward", "route_forward", "route_backward", "grouped_forward",
           "grouped_backward_data", "grouped_backward_weight", "combine_forward",
           "combine_backward", "ROUTE_MAX_EXPERTS", "ROUTE_MAX_SLOTS"]


def _pkg():
    from . import _dtype_code, _stream_ptr, _torch
    return _torch(), _dtype_code, _stream_ptr


def _on_stream(fn):
    """Run a call, its copies and its allocations on the stream it is given; the
    tensors it was given are not reused before that stream is done with them."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        torch = _pkg()[0]
        with torch.cuda.stream(stream):
            out = fn(*args, **kw)
        for t in list(args) + list(kw.values()):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
        return out
    return call


def _given(t, name, dtypes, shape=None):
    """A contiguous tensor on the current device, of one of the dtypes and of a
    shape whose None entries may be anything."""
    torch = _pkg()[0]
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a cuda tensor")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, needs one of {dtypes}")
    if shape is not None and (t.dim() != len(shape) or
                              any(w is not None and w != s for w, s in zip(shape, t.shape))):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, needs {shape}")
    return t.contiguous()


def _features(torch):
    return (torch.float32, torch.bfloat16)


def _result(out, name, shape, dtype, device, inputs=()):
    """The output tensor: `out`, which must fit as it is, or a new one."""
    torch = _pkg()[0]
    if out is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if (not out.is_cuda or out.dtype != dtype or tuple(out.shape) != tuple(shape) or
            not out.is_contiguous() or out.device != device):
        raise ValueError(f"{name} must be a contiguous {dtype} cuda tensor of shape {tuple(shape)}")
    return out


def _ptr(t):
    return t.data_ptr() if t is not None and t.numel() else None


def _i32(t):
    """A host-side size as the C int it is passed as."""
    if t > 0x7fffffff:
        raise ValueError(f"size {t} is out of range")
    return int(t)


def _call(name, *args):
    _, _, stream_ptr = _pkg()
    _lib.check(getattr(_lib.load(), name)(*args, stream_ptr()), name)


def _workspace(name, device, *sizes):
    torch = _pkg()[0]
    n = ctypes.c_size_t()
    _lib.check(getattr(_lib.load(), name)(*sizes, ctypes.byref(n)), name)
    return (torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None), n.value


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
@_on_stream
def layer_norm_forward(x, gamma=None, beta=None, eps=1e-5, *, stats=True, out=None):
    """(y, mean, rstd) of the rows of x [n, C]: y = (x - mean) * rstd * gamma + beta, with gamma
    and beta float32 [C] or None.  mean and rstd (float32 [n]) are what layer_norm_backward
    needs; stats=False leaves them out (None)."""
    torch, code, _ = _pkg()
    x = _given(x, "x", _features(torch), (None, None))
    n, C = x.shape
    if gamma is not None:
        gamma = _given(gamma, "gamma", (torch.float32,), (C,))
    if beta is not None:
        beta = _given(beta, "beta", (torch.float32,), (C,))
    y = _result(out, "out", (n, C), x.dtype, x.device)
    mean = torch.empty(n, dtype=torch.float32, device=x.device) if stats else None
    rstd = torch.empty_like(mean) if stats else None
    _call("spconv_layer_norm_forward", code(x.dtype), _ptr(x), _ptr(gamma), _ptr(beta),
          float(eps), _ptr(y), _ptr(mean), _ptr(rstd), n, _i32(C))
    return y, mean, rstd


@_on_stream
def layer_norm_backward(dy, x, mean, rstd, gamma=None, *, params=None, out=None):
    """(dx, dgamma, dbeta) of layer_norm_forward.  params says whether dgamma and dbeta
    (float32 [C]) are wanted; by default they are if gamma is given."""
    torch, code, _ = _pkg()
    x = _given(x, "x", _features(torch), (None, None))
    n, C = x.shape
    dy = _given(dy, "dy", (x.dtype,), (n, C))
    mean = _given(mean, "mean", (torch.float32,), (n,))
    rstd = _given(rstd, "rstd", (torch.float32,), (n,))
    if gamma is not None:
        gamma = _given(gamma, "gamma", (torch.float32,), (C,))
    params = gamma is not None if params is None else params
    dx = _result(out, "out", (n, C), x.dtype, x.device)
    dg = db = ws = None
    nbytes = 0
    if params:
        dg = torch.empty(C, dtype=torch.float32, device=x.device)
        db = torch.empty_like(dg)
        ws, nbytes = _workspace("spconv_layer_norm_backward_workspace", x.device, n, _i32(C))
    _call("spconv_layer_norm_backward", code(x.dtype), _ptr(dy), _ptr(x), _ptr(mean), _ptr(rstd),
          _ptr(gamma), _ptr(dx), _ptr(dg), _ptr(db), n, _i32(C), _ptr(ws), nbytes)
    return dx, dg, db


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
def _dropout(name, x, p, seed, offset, residual, step, out):
    torch, code, _ = _pkg()
    x = _given(x, "x", _features(torch))
    args = []
    if name.endswith("forward"):
        if residual is not None:
            residual = _given(residual, "residual", (x.dtype,), tuple(x.shape))
        args = [_ptr(residual)]
    if step is not None:
        step = _given(step, "step", (torch.int64,))
        if step.numel() != 1:
            raise ValueError("step must be one int64")
    y = _result(out, "out", tuple(x.shape), x.dtype, x.device)
    _call(name, code(x.dtype), _ptr(x), *args, float(p), int(seed) & 0xffffffffffffffff,
          int(offset) & 0xffffffffffffffff, _ptr(step), _ptr(y), x.numel())
    return y


@_on_stream
def dropout_forward(x, p, seed, offset=0, *, residual=None, step=None, out=None):
    """residual + (x / (1 - p) where the element is kept, else 0); element i (in flat order) is
    kept by word i % 4 of Philox4x32-7 for the counter (i / 4, offset) under the key `seed`.
    Another layer or step takes another offset; step, an int64 cuda tensor of one element, is
    added to it on the device (for captured graphs).  out may be x or residual."""
    return _dropout("spconv_dropout_forward", x, p, seed, offset, residual, step, out)


@_on_stream
def dropout_backward(dy, p, seed, offset=0, *, step=None, out=None):
    """Gradient of dropout_forward with respect to x (that of the residual is dy)."""
    return _dropout("spconv_dropout_backward", dy, p, seed, offset, None, step, out)


# ---------------------------------------------------------------------------
# Routing
# ---------------------------------------------------------------------------
class Routing:
    """Where every row goes.

    experts  int32 [n, k], largest logit first, -1 for none;  weights  float32 [n, k]
    offsets  int32 [E + 1]: expert e's pairs are positions offsets[e] .. offsets[e + 1]
    rows     int32 [n * k]: the row of every position, -1 from offsets[E] on
    pos      int32 [n, k]: the position of every (row, slot), -1 for none
    """

    __slots__ = ("experts", "weights", "offsets", "rows", "pos")

    def __init__(self, experts, weights, offsets, rows, pos):
        self.experts, self.weights, self.offsets = experts, weights, offsets
        self.rows, self.pos = rows, pos


@_on_stream
def route_forward(logits, k, normalize=True):
    """Send every row of logits [n, E] to the experts of its k largest logits (ties to the lowest
    expert; -inf is never chosen).  Weights are the softmax over the chosen (normalize=True) or
    the chosen entries of the softmax over all experts."""
    torch, code, _ = _pkg()
    logits = _given(logits, "logits", _features(torch), (None, None))
    n, E = logits.shape
    dev, k = logits.device, int(k)
    ws, nbytes = _workspace("spconv_route_workspace", dev, n, _i32(E), _i32(k))
    ints = functools.partial(torch.empty, dtype=torch.int32, device=dev)
    r = Routing(ints((n, k)), torch.empty((n, k), dtype=torch.float32, device=dev), ints(E + 1),
                ints(n * k), ints((n, k)))
    _call("spconv_route_forward", code(logits.dtype), _ptr(logits), n, E, k, 1 if normalize else 0,
          _ptr(r.experts), _ptr(r.weights), _ptr(r.offsets), _ptr(r.rows), _ptr(r.pos), _ptr(ws),
          nbytes)
    return r


@_on_stream
def route_backward(dweights, logits, experts, weights, normalize=True, *, out=None):
    """dlogits [n, E] (dtype of logits) from the gradient of the weights, float32 [n, k]."""
    torch, code, _ = _pkg()
    logits = _given(logits, "logits", _features(torch), (None, None))
    n, E = logits.shape
    dweights = _given(dweights, "dweights", (torch.float32,), (n, None))
    k = dweights.shape[1]
    experts = _given(experts, "experts", (torch.int32,), (n, k))
    weights = _given(weights, "weights", (torch.float32,), (n, k))
    d = _result(out, "out", (n, E), logits.dtype, logits.device)
    _call("spconv_route_backward", code(logits.dtype), _ptr(dweights), _ptr(logits), _ptr(experts),
          _ptr(weights), n, _i32(E), _i32(k), 1 if normalize else 0, _ptr(d))
    return d


# ---------------------------------------------------------------------------
# Grouped products
# ---------------------------------------------------------------------------
def _groups(torch, w, offsets, dtype):
    w = _given(w, "w", (dtype,), (None, None, None))
    return w, _given(offsets, "offsets", (torch.int32,), (w.shape[0] + 1,))


@_on_stream
def grouped_forward(x, w, offsets, *, rows=None, bias=None, relu=False, out_dtype=None, out=None):
    """y[j] = act(x[rows[j]] @ w[e] + bias[e]) for the positions offsets[e] <= j < offsets[e + 1]:
    x [n_x, C_in], w [E, C_in, C_out], offsets int32 [E + 1], rows int32 [m] or None (row j; m is
    then n_x), bias float32 [E, C_out] or None.  Positions from offsets[E] on are zero."""
    torch, code, _ = _pkg()
    x = _given(x, "x", _features(torch), (None, None))
    w, offsets = _groups(torch, w, offsets, x.dtype)
    E, ci, co = w.shape
    if x.shape[1] != ci:
        raise ValueError(f"x has {x.shape[1]} columns, w takes {ci}")
    if rows is not None:
        rows = _given(rows, "rows", (torch.int32,), (None,))
    if bias is not None:
        bias = _given(bias, "bias", (torch.float32,), (E, co))
    m = x.shape[0] if rows is None else rows.shape[0]
    out_dtype = x.dtype if out_dtype is None else out_dtype
    y = _result(out, "out", (m, co), out_dtype, x.device)
    _call("spconv_grouped_forward", code(x.dtype), _ptr(x), x.shape[0], _ptr(w), _ptr(offsets),
          _ptr(rows), _ptr(bias), 1 if relu else 0, code(out_dtype), _ptr(y), m, E, ci, co)
    return y


@_on_stream
def grouped_backward_data(dy, w, offsets, *, mask=None, out_dtype=None, out=None):
    """dx[j] = dy[j] @ w[e]^T per position, [m, C_in]; zero where mask [m, C_in] (of the output's
    dtype: the layer's input, if it came out of a ReLU) is <= 0.  For gathered rows,
    combine_forward(dx, pos) sums the positions of each row."""
    torch, code, _ = _pkg()
    dy = _given(dy, "dy", _features(torch), (None, None))
    w, offsets = _groups(torch, w, offsets, dy.dtype)
    E, ci, co = w.shape
    m = dy.shape[0]
    if dy.shape[1] != co:
        raise ValueError(f"dy has {dy.shape[1]} columns, w gives {co}")
    out_dtype = dy.dtype if out_dtype is None else out_dtype
    if mask is not None:
        mask = _given(mask, "mask", (out_dtype,), (m, ci))
    dx = _result(out, "out", (m, ci), out_dtype, dy.device)
    _call("spconv_grouped_backward_data", code(dy.dtype), _ptr(dy), _ptr(w), _ptr(offsets),
          _ptr(mask), code(out_dtype), _ptr(dx), m, E, ci, co)
    return dx


@_on_stream
def grouped_backward_weight(x, dy, offsets, *, rows=None, bias=True):
    """(dw float32 [E, C_in, C_out], db float32 [E, C_out] or None) of grouped_forward with the
    same x, offsets and rows."""
    torch, code, _ = _pkg()
    x = _given(x, "x", _features(torch), (None, None))
    dy = _given(dy, "dy", (x.dtype,), (None, None))
    offsets = _given(offsets, "offsets", (torch.int32,), (None,))
    E, ci, co, m = offsets.shape[0] - 1, x.shape[1], dy.shape[1], dy.shape[0]
    if rows is not None:
        rows = _given(rows, "rows", (torch.int32,), (m,))
    elif x.shape[0] != m:
        raise ValueError(f"x has {x.shape[0]} rows, dy {m}")
    ws, nbytes = _workspace("spconv_grouped_backward_weight_workspace", x.device, code(x.dtype), m,
                            E, ci, co)
    dw = torch.empty((max(E, 0), ci, co), dtype=torch.float32, device=x.device)
    db = torch.empty((max(E, 0), co), dtype=torch.float32, device=x.device) if bias else None
    _call("spconv_grouped_backward_weight", code(x.dtype), _ptr(x), x.shape[0], _ptr(dy),
          _ptr(offsets), _ptr(rows), _ptr(dw), _ptr(db), m, E, ci, co, _ptr(ws), nbytes)
    return dw, db


# ---------------------------------------------------------------------------
# Combine
# ---------------------------------------------------------------------------
@_on_stream
def combine_forward(y, pos, weights=None, *, residual=None, out=None):
    """out[i] = residual[i] + sum_s weights[i, s] * y[pos[i, s]]: y [m, C], pos int32 [n, k] (-1
    adds nothing), weights float32 [n, k] or None (ones).  out may be residual."""
    torch, code, _ = _pkg()
    y = _given(y, "y", _features(torch), (None, None))
    m, C = y.shape
    pos = _given(pos, "pos", (torch.int32,), (None, None))
    n, k = pos.shape
    if weights is not None:
        weights = _given(weights, "weights", (torch.float32,), (n, k))
    if residual is not None:
        residual = _given(residual, "residual", (y.dtype,), (n, C))
    o = _result(out, "out", (n, C), y.dtype, y.device)
    _call("spconv_combine_forward", code(y.dtype), _ptr(y), m, _ptr(pos), _ptr(weights),
          _ptr(residual), _ptr(o), n, _i32(k), _i32(C))
    return o


@_on_stream
def combine_backward(dout, y, pos, weights=None, *, offsets=None, out=None):
    """(dy [m, C], dweights float32 [n, k] or None without weights) of combine_forward (that of
    the residual is dout).  offsets: the routing's, whose last entry says from where on dy is
    zero; None if pos refers to every row of y."""
    torch, code, _ = _pkg()
    y = _given(y, "y", _features(torch), (None, None))
    m, C = y.shape
    pos = _given(pos, "pos", (torch.int32,), (None, None))
    n, k = pos.shape
    dout = _given(dout, "dout", (y.dtype,), (n, C))
    dw = None
    if weights is not None:
        weights = _given(weights, "weights", (torch.float32,), (n, k))
        dw = torch.empty((n, k), dtype=torch.float32, device=y.device)
    count = None
    if offsets is not None:
        offsets = _given(offsets, "offsets", (torch.int32,), (None,))
        if offsets.shape[0] < 1:
            raise ValueError("offsets is empty")
        count = offsets.data_ptr() + 4 * (offsets.shape[0] - 1)
    dy = _result(out, "out", (m, C), y.dtype, y.device)
    _call("spconv_combine_backward", code(y.dtype), _ptr(dout), _ptr(y), _ptr(pos), _ptr(weights),
          count, _ptr(dy), _ptr(dw), m, n, _i32(k), _i32(C))
    return dy, dw
