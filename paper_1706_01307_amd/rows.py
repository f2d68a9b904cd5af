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

import ctypes
import functools

from . import _lib
from ._lib import BF16, F32, ROUTE_MAX_EXPERTS, ROUTE_MAX_SLOTS

__all__ = ["Routing", "layer_norm_forward", "layer_norm_backward", "dropout_forward",
           "dropout_backward", "route_forward", "route_backward", "grouped_forward",
           "grouped_backward_data", "grouped_backward_weight", "combine_forward",
           "combine_backward", "ROUTE_MAX_EXPERTS", "ROUTE_MAX_SLOTS"]

# What every call needs, set by the first one (torch is imported late here): a
# call on a small tensor takes as long as its marshalling, so nothing is looked
# up twice.
torch = None
_CODE = {}                 # dtype -> code; the types features can have
_FLOAT = _INT = ()         # parameters' and indices' dtypes
_device = _raw_stream = _lib_fn = None


def _ready():
    global torch, _FLOAT, _INT, _device, _raw_stream, _lib_fn
    import torch as t
    lib = _lib.load()
    t.cuda.init()
    _device = t._C._cuda_getDevice
    _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (
        lambda dev: t.cuda.current_stream(dev).cuda_stream)
    _lib_fn = {name: getattr(lib, name) for name in _lib.ROWS_SIGNATURES}
    _CODE.update({t.float32: F32, t.bfloat16: BF16})
    _FLOAT, _INT = (t.float32,), (t.int32,)
    torch = t


def _on_stream(fn):
    """Run a call, its copies and its allocations on the stream it is given; the
    tensors it was given are not reused before that stream is done with them."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if torch is None:
            for t in args[:1]:
                if not getattr(t, "is_cuda", False):
                    raise TypeError("the first argument must be a cuda tensor")
            _ready()
        if stream is None:
            return fn(*args, **kw)
        with torch.cuda.stream(stream):
            out = fn(*args, **kw)
        for t in list(args) + list(kw.values()):
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
        return out
    return call


def _given(t, name, dtypes, shape, dims=0):
    """t, contiguous, if it is a cuda tensor on the current device, of one of the
    dtypes and of the shape (or, with shape None, of that many dimensions)."""
    if (type(t) is not torch.Tensor and not isinstance(t, torch.Tensor)) or not t.is_cuda:
        raise TypeError(f"{name} must be a cuda tensor")
    if t.get_device() != _device():
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, needs one of {tuple(dtypes)}")
    if t.shape != shape if shape is not None else dims and t.dim() != dims:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, needs "
                         f"{shape if shape is not None else f'{dims} dimensions'}")
    return t if t.is_contiguous() else t.contiguous()


def _result(out, shape, dtype, like):
    """The output tensor: `out`, which must fit as it is, or a new one beside `like`."""
    if out is None:
        if like.dtype == dtype and like.shape == shape:
            return torch.empty_like(like)          # (the quicker of the two)
        return torch.empty(shape, dtype=dtype, device=like.device)
    if (not isinstance(out, torch.Tensor) or out.device != like.device or out.dtype != dtype or
            out.shape != shape or not out.is_contiguous()):
        raise ValueError(f"out must be a contiguous {dtype} tensor of shape {tuple(shape)} on "
                         f"{like.device}")
    return out


def _ptr(t):
    return None if t is None else t.data_ptr()


def _i32(v):
    """A size as the C int it is passed as."""
    if v > 0x7fffffff:
        raise ValueError(f"size {v} is out of range")
    return v


def _call(name, *args):
    st = _lib_fn[name](*args, _raw_stream(_device()))
    if st:
        _lib.check(st, name)


def _workspace(name, like, *sizes):
    n = ctypes.c_size_t()
    st = _lib_fn[name](*sizes, ctypes.byref(n))
    if st:
        _lib.check(st, name)
    return (torch.empty(n.value, dtype=torch.uint8, device=like.device) if n.value else None,
            n.value)


# ---------------------------------------------------------------------------
# Layer norm
# ---------------------------------------------------------------------------
@_on_stream
def layer_norm_forward(x, gamma=None, beta=None, eps=1e-5, *, stats=True, out=None):
    """(y, mean, rstd) of the rows of x [n, C]: y = (x - mean) * rstd * gamma + beta, with gamma
    and beta float32 [C] or None.  mean and rstd (float32 [n]) are what layer_norm_backward
    needs; stats=False leaves them out (None)."""
    x = _given(x, "x", _CODE, None, 2)
    n, C = x.shape
    if gamma is not None:
        gamma = _given(gamma, "gamma", _FLOAT, (C,))
    if beta is not None:
        beta = _given(beta, "beta", _FLOAT, (C,))
    y = _result(out, (n, C), x.dtype, x)
    mean = torch.empty(n, dtype=torch.float32, device=x.device) if stats else None
    rstd = torch.empty_like(mean) if stats else None
    _call("spconv_layer_norm_forward", _CODE[x.dtype], _ptr(x), _ptr(gamma), _ptr(beta),
          float(eps), _ptr(y), _ptr(mean), _ptr(rstd), n, _i32(C))
    return y, mean, rstd


@_on_stream
def layer_norm_backward(dy, x, mean, rstd, gamma=None, *, params=None, out=None):
    """(dx, dgamma, dbeta) of layer_norm_forward.  params says whether dgamma and dbeta
    (float32 [C]) are wanted; by default they are if gamma is given."""
    x = _given(x, "x", _CODE, None, 2)
    n, C = x.shape
    dy = _given(dy, "dy", (x.dtype,), (n, C))
    mean = _given(mean, "mean", _FLOAT, (n,))
    rstd = _given(rstd, "rstd", _FLOAT, (n,))
    if gamma is not None:
        gamma = _given(gamma, "gamma", _FLOAT, (C,))
    params = gamma is not None if params is None else params
    dx = _result(out, (n, C), x.dtype, x)
    dg = db = ws = None
    nbytes = 0
    if params:
        dg = torch.empty(C, dtype=torch.float32, device=x.device)
        db = torch.empty_like(dg)
        ws, nbytes = _workspace("spconv_layer_norm_backward_workspace", x, n, _i32(C))
    _call("spconv_layer_norm_backward", _CODE[x.dtype], _ptr(dy), _ptr(x), _ptr(mean), _ptr(rstd),
          _ptr(gamma), _ptr(dx), _ptr(dg), _ptr(db), n, _i32(C), _ptr(ws), nbytes)
    return dx, dg, db


# ---------------------------------------------------------------------------
# Dropout
# ---------------------------------------------------------------------------
def _dropout(name, x, p, seed, offset, residual, step, out):
    x = _given(x, "x", _CODE, None)
    args = []
    if name.endswith("forward"):
        if residual is not None:
            residual = _given(residual, "residual", (x.dtype,), tuple(x.shape))
        args = [_ptr(residual)]
    if step is not None:
        step = _given(step, "step", (torch.int64,), None)
        if step.numel() != 1:
            raise ValueError("step must be one int64")
    y = _result(out, tuple(x.shape), x.dtype, x)
    _call(name, _CODE[x.dtype], _ptr(x), *args, float(p), int(seed) & 0xffffffffffffffff,
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
    logits = _given(logits, "logits", _CODE, None, 2)
    n, E = logits.shape
    dev, k = logits.device, int(k)
    ws, nbytes = _workspace("spconv_route_workspace", logits, n, _i32(E), _i32(k))
    ints = functools.partial(torch.empty, dtype=torch.int32, device=dev)
    r = Routing(ints((n, k)), torch.empty((n, k), dtype=torch.float32, device=dev), ints(E + 1),
                ints(n * k), ints((n, k)))
    _call("spconv_route_forward", _CODE[logits.dtype], _ptr(logits), n, E, k, 1 if normalize else 0,
          _ptr(r.experts), _ptr(r.weights), _ptr(r.offsets), _ptr(r.rows), _ptr(r.pos), _ptr(ws),
          nbytes)
    return r


@_on_stream
def route_backward(dweights, logits, experts, weights, normalize=True, *, out=None):
    """dlogits [n, E] (dtype of logits) from the gradient of the weights, float32 [n, k]."""
    logits = _given(logits, "logits", _CODE, None, 2)
    n, E = logits.shape
    dweights = _given(dweights, "dweights", _FLOAT, None, 2)
    k = dweights.shape[1]
    if dweights.shape[0] != n:
        raise ValueError(f"dweights has {dweights.shape[0]} rows, logits {n}")
    experts = _given(experts, "experts", _INT, (n, k))
    weights = _given(weights, "weights", _FLOAT, (n, k))
    d = _result(out, (n, E), logits.dtype, logits)
    _call("spconv_route_backward", _CODE[logits.dtype], _ptr(dweights), _ptr(logits), _ptr(experts),
          _ptr(weights), n, _i32(E), _i32(k), 1 if normalize else 0, _ptr(d))
    return d


# ---------------------------------------------------------------------------
# Grouped products
# ---------------------------------------------------------------------------
def _groups(w, offsets, dtype):
    w = _given(w, "w", (dtype,), None, 3)
    for size in w.shape:
        _i32(size)
    return w, _given(offsets, "offsets", _INT, (w.shape[0] + 1,))


def _out_dtype(dtype, x):
    if dtype is None:
        return x.dtype
    if dtype not in _CODE:
        raise TypeError(f"unsupported dtype {dtype}: use float32 or bfloat16")
    return dtype


@_on_stream
def grouped_forward(x, w, offsets, *, rows=None, bias=None, relu=False, out_dtype=None, out=None):
    """y[j] = act(x[rows[j]] @ w[e] + bias[e]) for the positions offsets[e] <= j < offsets[e + 1]:
    x [n_x, C_in], w [E, C_in, C_out], offsets int32 [E + 1], rows int32 [m] or None (row j; m is
    then n_x), bias float32 [E, C_out] or None.  Positions from offsets[E] on are zero."""
    x = _given(x, "x", _CODE, None, 2)
    w, offsets = _groups(w, offsets, x.dtype)
    E, ci, co = w.shape
    if x.shape[1] != ci:
        raise ValueError(f"x has {x.shape[1]} columns, w takes {ci}")
    if rows is not None:
        rows = _given(rows, "rows", _INT, None, 1)
    if bias is not None:
        bias = _given(bias, "bias", _FLOAT, (E, co))
    m = x.shape[0] if rows is None else rows.shape[0]
    out_dtype = _out_dtype(out_dtype, x)
    y = _result(out, (m, co), out_dtype, x)
    _call("spconv_grouped_forward", _CODE[x.dtype], _ptr(x), x.shape[0], _ptr(w), _ptr(offsets),
          _ptr(rows), _ptr(bias), 1 if relu else 0, _CODE[out_dtype], _ptr(y), m, E, ci, co)
    return y


@_on_stream
def grouped_backward_data(dy, w, offsets, *, mask=None, out_dtype=None, out=None):
    """dx[j] = dy[j] @ w[e]^T per position, [m, C_in]; zero where mask [m, C_in] (of the output's
    dtype: the layer's input, if it came out of a ReLU) is <= 0.  For gathered rows,
    combine_forward(dx, pos) sums the positions of each row."""
    dy = _given(dy, "dy", _CODE, None, 2)
    w, offsets = _groups(w, offsets, dy.dtype)
    E, ci, co = w.shape
    m = dy.shape[0]
    if dy.shape[1] != co:
        raise ValueError(f"dy has {dy.shape[1]} columns, w gives {co}")
    out_dtype = _out_dtype(out_dtype, dy)
    if mask is not None:
        mask = _given(mask, "mask", (out_dtype,), (m, ci))
    dx = _result(out, (m, ci), out_dtype, dy)
    _call("spconv_grouped_backward_data", _CODE[dy.dtype], _ptr(dy), _ptr(w), _ptr(offsets),
          _ptr(mask), _CODE[out_dtype], _ptr(dx), m, E, ci, co)
    return dx


@_on_stream
def grouped_backward_weight(x, dy, offsets, *, rows=None, bias=True):
    """(dw float32 [E, C_in, C_out], db float32 [E, C_out] or None) of grouped_forward with the
    same x, offsets and rows."""
    x = _given(x, "x", _CODE, None, 2)
    dy = _given(dy, "dy", (x.dtype,), None, 2)
    offsets = _given(offsets, "offsets", _INT, None, 1)
    E, ci, co = _i32(offsets.shape[0] - 1), _i32(x.shape[1]), _i32(dy.shape[1])
    m = dy.shape[0]
    if rows is not None:
        rows = _given(rows, "rows", _INT, (m,))
    elif x.shape[0] != m:
        raise ValueError(f"x has {x.shape[0]} rows, dy {m}")
    ws, nbytes = _workspace("spconv_grouped_backward_weight_workspace", x, _CODE[x.dtype], m,
                            E, ci, co)
    dw = torch.empty((max(E, 0), ci, co), dtype=torch.float32, device=x.device)
    db = torch.empty((max(E, 0), co), dtype=torch.float32, device=x.device) if bias else None
    _call("spconv_grouped_backward_weight", _CODE[x.dtype], _ptr(x), x.shape[0], _ptr(dy),
          _ptr(offsets), _ptr(rows), _ptr(dw), _ptr(db), m, E, ci, co, _ptr(ws), nbytes)
    return dw, db


# ---------------------------------------------------------------------------
# Combine
# ---------------------------------------------------------------------------
@_on_stream
def combine_forward(y, pos, weights=None, *, residual=None, out=None):
    """out[i] = residual[i] + sum_s weights[i, s] * y[pos[i, s]]: y [m, C], pos int32 [n, k] (-1
    adds nothing), weights float32 [n, k] or None (ones).  out may be residual."""
    y = _given(y, "y", _CODE, None, 2)
    m, C = y.shape
    pos = _given(pos, "pos", _INT, None, 2)
    n, k = pos.shape
    if weights is not None:
        weights = _given(weights, "weights", _FLOAT, (n, k))
    if residual is not None:
        residual = _given(residual, "residual", (y.dtype,), (n, C))
    o = _result(out, (n, C), y.dtype, y)
    _call("spconv_combine_forward", _CODE[y.dtype], _ptr(y), m, _ptr(pos), _ptr(weights),
          _ptr(residual), _ptr(o), n, _i32(k), _i32(C))
    return o


@_on_stream
def combine_backward(dout, y, pos, weights=None, *, offsets=None, out=None):
    """(dy [m, C], dweights float32 [n, k] or None without weights) of combine_forward (that of
    the residual is dout).  offsets: the routing's, whose last entry says from where on dy is
    zero; None if pos refers to every row of y."""
    y = _given(y, "y", _CODE, None, 2)
    m, C = y.shape
    pos = _given(pos, "pos", _INT, None, 2)
    n, k = pos.shape
    dout = _given(dout, "dout", (y.dtype,), (n, C))
    dw = None
    if weights is not None:
        weights = _given(weights, "weights", _FLOAT, (n, k))
        dw = torch.empty((n, k), dtype=torch.float32, device=y.device)
    count = None
    if offsets is not None:
        offsets = _given(offsets, "offsets", _INT, None, 1)
        if offsets.shape[0] < 1:
            raise ValueError("offsets is empty")
        count = offsets.data_ptr() + 4 * (offsets.shape[0] - 1)
    dy = _result(out, (m, C), y.dtype, y)
    _call("spconv_combine_backward", _CODE[y.dtype], _ptr(dout), _ptr(y), _ptr(pos), _ptr(weights),
          count, _ptr(dy), _ptr(dw), m, n, _i32(k), _i32(C))
    return dy, dw
