"""Python binding of the sequence operators of libtq (include/tq_seq.h):
argument marshalling only.

Operators of sequence models over measurement records: embedding of the
sampler's bitstrings, the gated linear recurrence over time, layer norm and
the softmax cross entropy over the vocabulary of bitstrings, each with its
gradient.  Tensors live on the current HIP device; ids are int64, the bit
patterns of the uint64 ids of the library, so that -1 is the marker of a
missing shot.  Outputs and workspaces that the caller does not give come from
torch's allocator for the stream the call runs on.
"""
import ctypes
import functools

import torch

from . import tq

SCAN_PIECE = 64  # TQ_SCAN_PIECE: steps per state that gated_scan keeps for its gradient

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_lib = None


def lib():
    """libtq.so with the prototypes of tq_seq.h."""
    global _lib
    if _lib is None:
        L = tq.lib()
        vp, i32, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        need = ctypes.POINTER(sz)
        protos = {
            "tq_embed": [vp, i64, i32, i64, i64, vp, i64, f32, vp, i64, vp],
            "tq_embed_grad_workspace": [i64, i64, i64, need],
            "tq_embed_grad": [vp, i64, i32, i64, i64, vp, i64, f32, vp, i64, vp, sz, vp],
            "tq_gated_scan_workspace": [i64, i64, i64, need],
            "tq_gated_scan": [i32, i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, vp, vp, i64, i64, vp, vp, vp, sz, vp],
            "tq_gated_scan_grad": [i32, i64, i64, i64, vp, i64, i64, vp, i64, i64, vp, vp, vp, i64, i64, vp, vp, i64, i64,
                                   vp, i64, i64, vp, vp, sz, vp],
            "tq_layer_norm": [vp, i64, i32, i64, i64, vp, vp, f32, vp, i64, vp, vp, vp],
            "tq_layer_norm_grad_workspace": [i64, i64, need],
            "tq_layer_norm_grad": [vp, i64, i32, i64, i64, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp],
            "tq_softmax_xent_workspace": [i32, i64, i64, i64, need],
            "tq_softmax_xent": [vp, i64, i32, i64, i64, i64, vp, i64, vp, vp, vp, vp, sz, vp],
            "tq_softmax_xent_grad_workspace": [i32, i64, i64, i64, need],
            "tq_softmax_xent_grad": [vp, i64, i32, i64, i64, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp, vp, sz, vp],
        }
        for name, args in protos.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        _lib = L
    return _lib


# ------------------------------------------------------------------ arguments
# The smallest calls are all latency: what runs on every call is kept short.

_raw_stream = torch._C._cuda_getCurrentRawStream
_device = torch._C._cuda_getDevice
_many = torch.cuda.device_count() > 1  # else there is no other device to be on


def _call(f, *args):
    rc = f(*args)
    if rc:
        raise tq.TQError(rc, lib().tq_last_error().decode())


def _tensor(t, name, dtype=None, shape=None):
    """t, checked to be on the current device, of `dtype` and `shape`."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if _many and t.get_device() != _device():
        raise ValueError(f"{name} is on device {t.get_device()}, the current device is {_device()}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return t


def _typed(t, name):
    """The type code of t and the device the call runs on, t's, which has to be
    the current one."""
    _tensor(t, name)
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code, t.get_device()


def _dense(t, name, dtype, shape=None):
    """Pointer of a contiguous tensor, None for None."""
    if t is None:
        return None
    _tensor(t, name, dtype, shape)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(t, name, dtype=None, shape=None):
    """(pointer, distance of rows) of a tensor whose last axis is contiguous and
    whose other axes run through rows at one distance."""
    _tensor(t, name, dtype, shape)
    if t.dim() < 1:
        raise ValueError(f"{name} must have one dimension at least")
    D = t.shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), D
    st = t.stride()
    ok = st[-1] == 1 or D <= 1
    step = None
    for k in range(t.dim() - 2, -1, -1):
        if t.shape[k] == 1:
            continue
        if step is None:
            step = reach = st[k]
        ok = ok and st[k] == reach
        reach = st[k] * t.shape[k]
    step = D if step is None else step
    if not ok or step < D:
        raise ValueError(f"{name} must be contiguous along its last axis with its rows at one distance")
    return t.data_ptr(), step


def _steps(t, name, dtype, shape):
    """(pointer, batch stride, step stride) of a [B, T, D] tensor."""
    _tensor(t, name, dtype, shape)
    sb, ss, sd = t.stride()
    if sd != 1 and shape[2] > 1 and t.numel():
        raise ValueError(f"{name} must be contiguous along its last axis")
    return t.data_ptr(), sb, ss


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on_stream(f):
    """Gives f's `stream` argument as a raw handle.  A stream other than torch's
    current one is made current while f allocates, so that the allocator ties
    what it gives to that stream."""
    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        if stream is None:
            return f(*args, **kw)
        with torch.cuda.stream(stream):
            return f(*args, **kw)
    return call


@functools.lru_cache(maxsize=256)
def _need(fn, *sizes):
    """Bytes of workspace that the library asks for with these sizes."""
    need = ctypes.c_size_t()
    _call(getattr(lib(), fn), *sizes, ctypes.byref(need))
    return need.value


def _space(like, n):
    return torch.empty(n, dtype=torch.uint8, device=like.device) if n else None


# ------------------------------------------------------------------ embedding

@_on_stream
def embed(tokens, table, scale=1.0, out=None):
    """scale * table[tokens] (tq_embed): tokens int64 of any shape, table
    [V, D]; a token outside the table (-1: no shot) gives a row of zeros."""
    code, dev = _typed(table, "table")
    if table.dim() != 2:
        raise ValueError("table must be [V, D]")
    kp = _dense(tokens, "tokens", torch.int64)
    tp, ld = _rows(table, "table")
    V, D = table.shape
    if out is None:
        out = table.new_empty(tokens.shape + (D,))
        op, ldo = out.data_ptr(), D
    else:
        op, ldo = _rows(out, "out", table.dtype, tokens.shape + (D,))
    _call((_lib or lib()).tq_embed, tp, ld, code, V, D, kp, tokens.numel(), scale, op, ldo, _raw_stream(dev))
    return out


@_on_stream
def embed_grad(tokens, grad_out, vocab, scale=1.0, grad=None):
    """Gradient [vocab, D] of embed's table from that of its output
    (tq_embed_grad); bitwise reproducible."""
    code, dev = _typed(grad_out, "grad_out")
    kp = _dense(tokens, "tokens", torch.int64)
    if grad_out.dim() < 1 or grad_out.shape[:-1] != tokens.shape:
        raise ValueError(f"grad_out must have shape {tuple(tokens.shape)} + [D], got {tuple(grad_out.shape)}")
    gp, ld = _rows(grad_out, "grad_out")
    D, N = grad_out.shape[-1], tokens.numel()
    if grad is None:
        grad = grad_out.new_empty((vocab, D))
        op, ldo = grad.data_ptr(), D
    else:
        op, ldo = _rows(grad, "grad", grad_out.dtype, (vocab, D))
    n = _need("tq_embed_grad_workspace", vocab, D, N)
    ws = _space(grad_out, n)
    _call((_lib or lib()).tq_embed_grad, gp, ld, code, vocab, D, kp, N, scale, op, ldo, _ptr(ws), n, _raw_stream(dev))
    return grad


# ----------------------------------------------------------------- recurrence

def _scan_shape(x, g, lengths):
    code, dev = _typed(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be a [B, T, D] tensor")
    shape = x.shape
    return (code, dev, shape, _steps(x, "x", None, shape) + _steps(g, "g", x.dtype, shape),
            _dense(lengths, "lengths", torch.int32, shape[:1]))


def _steps_out(t, name, x):
    """A given output of x's shape, or a new one: (tensor, its steps)."""
    if t is None:
        t = x.new_empty(x.shape)
    return t, _steps(t, name, x.dtype, x.shape)


@_on_stream
def gated_scan(x, g, h0=None, lengths=None, keep=False, y=None, h_last=None, states=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(g_t) over the steps
    of x, g [B, T, D] (tq_gated_scan), from h0 float32 [B, D] (None: zeros);
    lengths int32 [B] (None: all T).  Returns (y, h_last), with keep=True
    (y, h_last, states), the states being what gated_scan_grad needs.  h_last
    may be the h0 tensor: the records' states then advance in place."""
    code, dev, shape, xg, lp = _scan_shape(x, g, lengths)
    B, T, D = shape
    hp = _dense(h0, "h0", torch.float32, (B, D))
    y, ys = _steps_out(y, "y", x)
    if h_last is None:
        h_last = torch.empty((B, D), dtype=torch.float32, device=x.device)
    pieces = -(-T // SCAN_PIECE)
    if states is None and keep:
        states = torch.empty((B, pieces, D), dtype=torch.float32, device=x.device)
    n = _need("tq_gated_scan_workspace", B, T, D)
    ws = _space(x, n)
    _call((_lib or lib()).tq_gated_scan, code, B, T, D, *xg, hp, lp, *ys,
          _dense(h_last, "h_last", torch.float32, (B, D)), _dense(states, "states", torch.float32, (B, pieces, D)),
          _ptr(ws), n, _raw_stream(dev))
    return (y, h_last, states) if states is not None else (y, h_last)


@_on_stream
def gated_scan_grad(x, g, states, dy, dh_last=None, lengths=None, dx=None, dg=None, dh0=None):
    """(dx, dg, dh0) from the gradients of gated_scan's y and h_last (None:
    zeros) and the states it kept (tq_gated_scan_grad)."""
    code, dev, shape, xg, lp = _scan_shape(x, g, lengths)
    B, T, D = shape
    sp = _dense(states, "states", torch.float32, (B, -(-T // SCAN_PIECE), D))
    dp = _dense(dh_last, "dh_last", torch.float32, (B, D))
    dys = _steps(dy, "dy", x.dtype, shape)
    dx, dxs = _steps_out(dx, "dx", x)
    dg, dgs = _steps_out(dg, "dg", x)
    if dh0 is None:
        dh0 = torch.empty((B, D), dtype=torch.float32, device=x.device)
    n = _need("tq_gated_scan_workspace", B, T, D)
    ws = _space(x, n)
    _call((_lib or lib()).tq_gated_scan_grad, code, B, T, D, *xg, sp, lp, *dys, dp, *dxs, *dgs,
          _dense(dh0, "dh0", torch.float32, (B, D)), _ptr(ws), n, _raw_stream(dev))
    return dx, dg, dh0


# ----------------------------------------------------------------- layer norm

def _rows_out(t, name, x):
    """A given output of x's shape, or a new one: (tensor, pointer, distance of rows)."""
    if t is None:
        t = x.new_empty(x.shape)
        return t, t.data_ptr(), x.shape[-1]
    return (t,) + _rows(t, name, x.dtype, x.shape)


@_on_stream
def layer_norm(x, weight, bias=None, eps=1e-5, keep=False, y=None):
    """Layer norm over the last axis of x (tq_layer_norm): y, or with keep=True
    (y, mean, rstd), the latter two float32 as layer_norm_grad needs them."""
    code, dev = _typed(x, "x")
    xp, ld = _rows(x, "x")
    D = x.shape[-1]
    wp = _dense(weight, "weight", x.dtype, (D,))
    bp = _dense(bias, "bias", x.dtype, (D,))
    y, yp, ldy = _rows_out(y, "y", x)
    mean = rstd = None
    if keep:
        mean, rstd = torch.empty((2,) + x.shape[:-1], dtype=torch.float32, device=x.device)
        if not D:  # of no values
            mean.fill_(float("nan")), rstd.fill_(float("nan"))
    _call((_lib or lib()).tq_layer_norm, xp, ld, code, x.numel() // D if D else 0, D, wp, bp, eps, yp, ldy, _ptr(mean),
          _ptr(rstd), _raw_stream(dev))
    return (y, mean, rstd) if keep else y


@_on_stream
def layer_norm_grad(x, weight, mean, rstd, dy, dx=None):
    """(dx, dweight, dbias) of layer_norm (tq_layer_norm_grad)."""
    code, dev = _typed(x, "x")
    xp, ld = _rows(x, "x")
    D = x.shape[-1]
    N = x.numel() // D if D else 0
    wp = _dense(weight, "weight", x.dtype, (D,))
    mp = _dense(mean, "mean", torch.float32, x.shape[:-1])
    rp = _dense(rstd, "rstd", torch.float32, x.shape[:-1])
    dyp, ld_dy = _rows(dy, "dy", x.dtype, x.shape)
    dx, dxp, ld_dx = _rows_out(dx, "dx", x)
    dw, db = x.new_empty((D,)), x.new_empty((D,))
    n = _need("tq_layer_norm_grad_workspace", N, D)
    ws = _space(x, n)
    _call((_lib or lib()).tq_layer_norm_grad, xp, ld, code, N, D, wp, mp, rp, dyp, ld_dy, dxp, ld_dx, dw.data_ptr(),
          db.data_ptr(), _ptr(ws), n, _raw_stream(dev))
    return dx, dw, db


# -------------------------------------------------------------- cross entropy

def _xent_args(hidden, weight, targets):
    code, dev = _typed(hidden, "hidden")
    hp, ldh = _rows(hidden, "hidden")
    D = hidden.shape[-1]
    wp, ldw = _rows(weight, "weight", hidden.dtype)
    if weight.dim() != 2 or weight.shape[1] != D:
        raise ValueError(f"weight must have shape [V, {D}], got {tuple(weight.shape)}")
    tp = _dense(targets, "targets", torch.int64, hidden.shape[:-1])
    return dev, (code, targets.numel(), weight.shape[0], D), hp, ldh, wp, ldw, tp


def _two(like, shape):
    a = torch.empty((2,) + shape, dtype=torch.float32, device=like.device)
    return a[0], a[1]


@_on_stream
def softmax_xent(hidden, weight, targets, loss=None, lse=None):
    """(loss, lse) float32, of the shape of targets, of the logits
    hidden @ weight^T (tq_softmax_xent); the loss of a target outside the
    vocabulary is 0."""
    dev, sizes, hp, ldh, wp, ldw, tp = _xent_args(hidden, weight, targets)
    if loss is None and lse is None:
        loss, lse = _two(hidden, targets.shape)
    loss = torch.empty_like(lse) if loss is None else loss
    lse = torch.empty_like(loss) if lse is None else lse
    lp = _dense(loss, "loss", torch.float32, targets.shape)
    sp = _dense(lse, "lse", torch.float32, targets.shape)
    n = _need("tq_softmax_xent_workspace", *sizes)
    ws = _space(hidden, n)
    _call((_lib or lib()).tq_softmax_xent, hp, ldh, *sizes, wp, ldw, tp, lp, sp, _ptr(ws), n, _raw_stream(dev))
    return loss, lse


@_on_stream
def softmax_xent_grad(hidden, weight, targets, upstream, dhidden=None, dweight=None):
    """(dhidden, dweight, loss, lse): the gradients of sum(upstream * loss) and
    softmax_xent's outputs, from one call (tq_softmax_xent_grad)."""
    dev, sizes, hp, ldh, wp, ldw, tp = _xent_args(hidden, weight, targets)
    up = _dense(upstream, "upstream", torch.float32, targets.shape)
    dhidden, dhp, ld_dh = _rows_out(dhidden, "dhidden", hidden)
    dweight, dwp, ld_dw = _rows_out(dweight, "dweight", weight)
    loss, lse = _two(hidden, targets.shape)
    n = _need("tq_softmax_xent_grad_workspace", *sizes)
    ws = _space(hidden, n)
    _call((_lib or lib()).tq_softmax_xent_grad, hp, ldh, *sizes, wp, ldw, tp, up, dhp, ld_dh, dwp, ld_dw,
          loss.data_ptr(), lse.data_ptr(), _ptr(ws), n, _raw_stream(dev))
    return dhidden, dweight, loss, lse
