"""Operators on feature rows, as used between sparse convolutions.

    y, mean, rstd = layer_norm_forward(x, gamma, beta)
    r = route_forward(logits, k)                               # r.rows, r.offsets, r.pos, ...
    h = grouped_forward(y, w1, r.offsets, rows=r.rows, bias=b1, relu=True)
    z = grouped_forward(h, w2, r.offsets, bias=b2)
    u = combine_forward(z, r.pos, r.weights)
    out = dropout_forward(u, 0.1, seed, offset=step, residual=x)

    n8, h, rstd = rms_norm_forward(x, gamma, residual=stream, packed=True)   # Rows8
    y, z = linear_forward(n8, w, bias, act="gelu", pre=True)
    r = route_scores_forward(logits, k, bias=balance, groups=8, top_groups=4)
    z8 = pack_rows(z)                                          # kept for the backward pass
    dz = linear_backward_data(dy2, w2, act="gelu", pre=z8)
    dw, db = linear_backward_weight(n8, dz)

Argument marshalling only (the C ABI is include/spconv_rows.h).  Tensors are on
torch's current device; inputs that are not contiguous are copied.  Everything,
copies included, runs on torch's current stream or on `stream`; tensors made on
another stream are the caller's to order, as for torch's own operators.
"""
from __future__ import annotations

import ctypes
import functools

from . import _lib
from ._lib import (ACTIVATIONS, BF16, E4M3, F32, ROUTE_MAX_EXPERTS, ROUTE_MAX_GROUPS,
                   ROUTE_MAX_SLOTS, SCORES)

__all__ = ["Routing", "layer_norm_forward", "layer_norm_backward", "dropout_forward",
           "dropout_backward", "route_forward", "route_backward", "grouped_forward",
           "grouped_backward_data", "grouped_backward_weight", "combine_forward",
           "combine_backward", "Rows8", "rms_norm_forward", "rms_norm_backward", "pack_rows",
           "unpack_rows", "activation_backward", "linear_forward", "linear_backward_data",
           "linear_backward_weight", "route_scores_forward", "route_scores_backward",
           "ROUTE_MAX_EXPERTS", "ROUTE_MAX_SLOTS", "ROUTE_MAX_GROUPS"]

# What every call needs, set by the first one (torch is imported late here): a
# call on a small tensor takes as long as its marshalling, so nothing is looked
# up twice.
torch = None
_CODE = {}                 # dtype -> code; the types features can have
_FLOAT = _INT = _E4M3 = () # parameters', indices' and 8-bit values' dtypes
_device = _raw_stream = _lib_fn = None


def _ready():
    global torch, _FLOAT, _INT, _E4M3, _device, _raw_stream, _lib_fn
    import torch as t
    lib = _lib.load()
    t.cuda.init()
    _device = t._C._cuda_getDevice
    _raw_stream = getattr(t._C, "_cuda_getCurrentRawStream", None) or (
        lambda dev: t.cuda.current_stream(dev).cuda_stream)
    _lib_fn = {name: getattr(lib, name) for name in _lib.ROWS_SIGNATURES}
    _CODE.update({t.float32: F32, t.bfloat16: BF16})
    _FLOAT, _INT, _E4M3 = (t.float32,), (t.int32,), (t.float8_e4m3fn,)
    torch = t


def _on_stream(fn):
    """Run a call, its copies and its allocations on the stream it is given; the
    tensors it was given are not reused before that stream is done with them."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if torch is None:
            for t in args[:1]:
                if not getattr(getattr(t, "q", t), "is_cuda", False):
                    raise TypeError("the first argument must be a cuda tensor")
            _ready()
        if stream is None:
            return fn(*args, **kw)
        with torch.cuda.stream(stream):
            out = fn(*args, **kw)
        for t in list(args) + list(kw.values()):
            for t in (t.q, t.scale) if isinstance(t, Rows8) else (t,):
                if isinstance(t, torch.Tensor) and t.is_cuda:
                    t.record_stream(stream)
        return out
    return call


def _given(t, name, dtypes, shape, dims=0):
    """t, contiguous, if it is a cuda tensor on the current device, of one of the
    dtypes and of the shape (or, with shape None, of that many dimensions)."""
    if type(t) is not torch.Tensor and not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a cuda tensor")
    if t.get_device() != _device():
        if not t.is_cuda:
            raise TypeError(f"{name} must be a cuda tensor")
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
        return like.new_empty(shape, dtype=dtype)
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
    return like.new_empty(n.value, dtype=torch.uint8) if n.value else None, n.value


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


# ---------------------------------------------------------------------------
# Rows in 8 bits
# ---------------------------------------------------------------------------
class Rows8:
    """Rows kept in 8 bits: they stand for q * scale.

    q      float8_e4m3fn [n, C];  scale  float32 [n]
    """

    __slots__ = ("q", "scale")

    def __init__(self, q, scale):
        self.q, self.scale = q, scale


def _given8(r, name, shape=None):
    """(q, scale) of Rows8, contiguous, of the shape (or of two dimensions)."""
    if not isinstance(r, Rows8):
        raise TypeError(f"{name} must be Rows8")
    q = _given(r.q, f"{name}.q", _E4M3, shape, 2)
    return q, _given(r.scale, f"{name}.scale", _FLOAT, (q.shape[0],))


def _either(t, name, dtypes, shape=None):
    """(tensor, scales or None, type's code) of a tensor of two dimensions or of Rows8."""
    if isinstance(t, Rows8):
        q, scale = _given8(t, name, shape)
        return q, scale, E4M3
    t = _given(t, name, dtypes, shape, 2)
    return t, None, _CODE[t.dtype]


def _act(act):
    if act not in ACTIVATIONS:
        raise ValueError(f"unknown activation {act!r}: use one of {tuple(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _new8(n, C, like):
    return Rows8(like.new_empty((n, C), dtype=torch.float8_e4m3fn),
                 like.new_empty(n, dtype=torch.float32))


@_on_stream
def pack_rows(x):
    """Rows8 of x [n, C]: e4m3 values with a scale a row, the row's largest magnitude / 448.  A row
    with an infinity or NaN stands for NaN."""
    x = _given(x, "x", _CODE, None, 2)
    n, C = x.shape
    r = _new8(n, C, x)
    _call("spconv_pack_rows", _CODE[x.dtype], _ptr(x), _ptr(r.q), _ptr(r.scale), n, _i32(C))
    return r


@_on_stream
def unpack_rows(r, dtype=None, *, act=None, out=None):
    """act(q * scale), [n, C] of dtype (bfloat16 by default): act None, "relu", "gelu" or "silu"."""
    q, scale = _given8(r, "r")
    n, C = q.shape
    dtype = _out_dtype(torch.bfloat16 if dtype is None else dtype, q)
    y = _result(out, (n, C), dtype, q)
    _call("spconv_unpack_rows", _ptr(q), _ptr(scale), _act(act), _CODE[dtype], _ptr(y), n, _i32(C))
    return y


@_on_stream
def activation_backward(dy, pre, act, *, out=None):
    """dy * act'(pre): pre, the activation's input, of dy's dtype or Rows8.  out may be dy."""
    dy = _given(dy, "dy", _CODE, None, 2)
    n, C = dy.shape
    pre, scale, code = _either(pre, "pre", (dy.dtype,), (n, C))
    dz = _result(out, (n, C), dy.dtype, dy)
    _call("spconv_activation_backward", _CODE[dy.dtype], _ptr(dy), code, _ptr(pre), _ptr(scale),
          _act(act), _ptr(dz), n, _i32(C))
    return dz


# ---------------------------------------------------------------------------
# Root-mean-square norm
# ---------------------------------------------------------------------------
@_on_stream
def rms_norm_forward(x, gamma=None, eps=1e-6, *, residual=None, packed=False, stats=True, out=None,
                     sum_out=None):
    """(y, h, rstd): h = x + residual in x's dtype (x itself without a residual) and
    y = h / sqrt(mean of h^2 + eps) * gamma, in x's dtype or, packed, as Rows8; gamma float32 [C] or
    None.  h and rstd (float32 [n]; None with stats=False) are what rms_norm_backward needs.
    sum_out (for h) may be x or residual; out is for y where it is not packed."""
    x = _given(x, "x", _CODE, None, 2)
    n, C = x.shape
    h = x
    if residual is not None:
        residual = _given(residual, "residual", (x.dtype,), (n, C))
        h = _result(sum_out, (n, C), x.dtype, x)
    elif sum_out is not None:
        raise ValueError("sum_out without a residual")
    if gamma is not None:
        gamma = _given(gamma, "gamma", _FLOAT, (C,))
    if packed:
        if out is not None:
            raise ValueError("out is for an output that is not packed")
        y = _new8(n, C, x)
        yp, ys, code = _ptr(y.q), _ptr(y.scale), E4M3
    else:
        y = _result(out, (n, C), x.dtype, x)
        yp, ys, code = _ptr(y), None, _CODE[x.dtype]
    rstd = x.new_empty(n, dtype=torch.float32) if stats else None
    _call("spconv_rms_norm_forward", _CODE[x.dtype], _ptr(x), _ptr(residual), _ptr(gamma),
          float(eps), None if residual is None else _ptr(h), code, yp, ys, _ptr(rstd), n, _i32(C))
    return y, h, rstd


@_on_stream
def rms_norm_backward(dy, h, rstd, gamma=None, *, dh=None, params=None, out=None):
    """(dx, dgamma) of rms_norm_forward: dx, of dy's dtype, is the gradient of x and of the
    residual; h of that dtype or Rows8; dh what reaches h past the norm.  params says whether dgamma
    (float32 [C]) is wanted; by default it is if gamma is given."""
    dy = _given(dy, "dy", _CODE, None, 2)
    n, C = dy.shape
    h, scale, code = _either(h, "h", (dy.dtype,), (n, C))
    rstd = _given(rstd, "rstd", _FLOAT, (n,))
    if gamma is not None:
        gamma = _given(gamma, "gamma", _FLOAT, (C,))
    if dh is not None:
        dh = _given(dh, "dh", (dy.dtype,), (n, C))
    params = gamma is not None if params is None else params
    dx = _result(out, (n, C), dy.dtype, dy)
    dg = ws = None
    nbytes = 0
    if params:
        dg = dy.new_empty(C, dtype=torch.float32)
        ws, nbytes = _workspace("spconv_rms_norm_backward_workspace", dy, n, _i32(C))
    _call("spconv_rms_norm_backward", _CODE[dy.dtype], _ptr(dy), code, _ptr(h), _ptr(scale),
          _ptr(rstd), _ptr(gamma), _ptr(dh), _ptr(dx), _ptr(dg), n, _i32(C), _ptr(ws), nbytes)
    return dx, dg


# ---------------------------------------------------------------------------
# Dense products
# ---------------------------------------------------------------------------
@_on_stream
def linear_forward(x, w, bias=None, *, act=None, residual=None, pre=False, out_dtype=None,
                   out=None):
    """(y, z): z = x @ w + bias and y = act(z) + residual.  x [n, C_in] or Rows8, w [C_in, C_out] of
    x's dtype (bfloat16 for Rows8), bias float32 [C_out] or None, act None, "relu", "gelu" (its tanh
    form) or "silu", residual [n, C_out] of the output's dtype (x's by default, bfloat16 for Rows8)
    or None.  z is None unless pre is true.  out may be residual."""
    x, scale, code = _either(x, "x", _CODE)
    dtype = torch.bfloat16 if code == E4M3 else x.dtype
    w = _given(w, "w", (dtype,), None, 2)
    n, ci = x.shape
    co = w.shape[1]
    if w.shape[0] != ci:
        raise ValueError(f"x has {ci} columns, w takes {w.shape[0]}")
    if bias is not None:
        bias = _given(bias, "bias", _FLOAT, (co,))
    out_dtype = _out_dtype(dtype if out_dtype is None else out_dtype, x)
    if residual is not None:
        residual = _given(residual, "residual", (out_dtype,), (n, co))
    y = _result(out, (n, co), out_dtype, x)
    z = torch.empty_like(y) if pre else None
    _call("spconv_linear_forward", code, _ptr(x), _ptr(scale), _ptr(w), _ptr(bias), _act(act),
          _ptr(residual), _CODE[out_dtype], _ptr(y), _ptr(z), n, _i32(ci), _i32(co))
    return y, z


@_on_stream
def linear_backward_data(dy, w, *, act=None, pre=None, out_dtype=None, out=None):
    """dx = (dy @ w^T) * act'(pre), [n, C_in]: act is the activation that the product's input came
    out of and pre that activation's input, of the output's dtype (dy's by default) or Rows8."""
    dy = _given(dy, "dy", _CODE, None, 2)
    w = _given(w, "w", (dy.dtype,), None, 2)
    n, (ci, co) = dy.shape[0], w.shape
    if dy.shape[1] != co:
        raise ValueError(f"dy has {dy.shape[1]} columns, w gives {co}")
    out_dtype = _out_dtype(out_dtype, dy)
    scale, code = None, _CODE[out_dtype]
    if (pre is None) != (act is None):
        raise ValueError("act and pre go together")
    if pre is not None:
        pre, scale, code = _either(pre, "pre", (out_dtype,), (n, ci))
    dx = _result(out, (n, ci), out_dtype, dy)
    _call("spconv_linear_backward_data", _CODE[dy.dtype], _ptr(dy), _ptr(w), _act(act), code,
          _ptr(pre), _ptr(scale), _CODE[out_dtype], _ptr(dx), n, _i32(ci), _i32(co))
    return dx


@_on_stream
def linear_backward_weight(x, dy, *, bias=True):
    """(dw float32 [C_in, C_out], db float32 [C_out] or None) of linear_forward with the same x (of
    dy's dtype, or Rows8 with a bfloat16 dy)."""
    x, scale, code = _either(x, "x", _CODE)
    dy = _given(dy, "dy", (torch.bfloat16 if code == E4M3 else x.dtype,), None, 2)
    n, ci, co = x.shape[0], _i32(x.shape[1]), _i32(dy.shape[1])
    if dy.shape[0] != n:
        raise ValueError(f"x has {n} rows, dy {dy.shape[0]}")
    ws, nbytes = _workspace("spconv_linear_backward_weight_workspace", x, code, n, ci, co)
    dw = dy.new_empty((ci, co), dtype=torch.float32)
    db = dy.new_empty(co, dtype=torch.float32) if bias else None
    _call("spconv_linear_backward_weight", code, _ptr(x), _ptr(scale), _ptr(dy), _ptr(dw), _ptr(db),
          n, ci, co, _ptr(ws), nbytes)
    return dw, db


# ---------------------------------------------------------------------------
# Routing by scores
# ---------------------------------------------------------------------------
def _score(score):
    if score not in SCORES:
        raise ValueError(f"unknown score {score!r}: use one of {tuple(SCORES)}")
    return SCORES[score]


@_on_stream
def route_scores_forward(logits, k, *, score="sigmoid", bias=None, groups=1, top_groups=1,
                         normalize=True, scale=1.0):
    """Send every row of logits [n, E] to the experts of its k largest scores ("sigmoid" or
    "softmax") plus bias (float32 [E] or None; for the choice alone), from the top_groups of `groups`
    groups of adjacent experts whose two best add up to most.  Weights are the chosen scores, divided
    by their sum (normalize) and times scale.  Scores are compared as 64-bit arithmetic has them;
    ties to the lowest expert; an expert whose logit is -inf is never chosen."""
    logits = _given(logits, "logits", _CODE, None, 2)
    n, E = logits.shape
    if bias is not None:
        bias = _given(bias, "bias", _FLOAT, (E,))
    k = int(k)
    ws, nbytes = _workspace("spconv_route_workspace", logits, n, _i32(E), _i32(k))
    ints = functools.partial(logits.new_empty, dtype=torch.int32)
    experts = ints((n, k))
    r = Routing(experts, logits.new_empty((n, k), dtype=torch.float32), ints(E + 1), ints(n * k),
                torch.empty_like(experts))
    _call("spconv_route_scores_forward", _CODE[logits.dtype], _ptr(logits), _ptr(bias), n, E, k,
          _score(score), _i32(int(groups)), _i32(int(top_groups)), 1 if normalize else 0,
          float(scale), _ptr(r.experts), _ptr(r.weights), _ptr(r.offsets), _ptr(r.rows),
          _ptr(r.pos), _ptr(ws), nbytes)
    return r


@_on_stream
def route_scores_backward(dweights, logits, experts, weights, *, score="sigmoid", normalize=True,
                          scale=1.0, out=None):
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
    _call("spconv_route_scores_backward", _CODE[logits.dtype], _ptr(dweights), _ptr(logits),
          _ptr(experts), _ptr(weights), n, _i32(E), _i32(k), _score(score), 1 if normalize else 0,
          float(scale), _ptr(d))
    return d
