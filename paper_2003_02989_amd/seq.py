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

import torch

from . import tq
from .tq import _check, _dev

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

def _type(t, name):
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _on_device(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} is on device {t.get_device()}, the current device is {torch.cuda.current_device()}")


def _typed(t, dtype, name):
    _on_device(t, name)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _rows(t, name, dtype=None, shape=None):
    """(pointer, rows, width, distance of rows) of a tensor whose last axis is
    contiguous and whose other axes run through rows at one distance."""
    _on_device(t, name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.dim() < 1:
        raise ValueError(f"{name} must have one dimension at least")
    D = t.shape[-1]
    if t.is_contiguous():
        return t.data_ptr(), t.numel() // D if D else 0, D, D
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
    n = 1
    for k in t.shape[:-1]:
        n *= k
    return t.data_ptr(), n, D, step


def _steps(t, name, dtype, shape):
    """(pointer, batch stride, step stride) of a [B, T, D] tensor."""
    _typed(t, dtype, name)
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
    sb, ss, sd = t.stride()
    if sd != 1 and shape[2] > 1:
        raise ValueError(f"{name} must be contiguous along its last axis")
    return t.data_ptr(), sb, ss


def _ptr(t):
    return None if t is None else t.data_ptr()


class _On:
    """The stream of a call, made torch's current one while the call allocates
    (so that the allocator ties the memory to it)."""

    def __init__(self, stream):
        now = torch.cuda.current_stream()
        self.handle = (stream or now).cuda_stream
        self.ctx = None
        if stream is not None and stream.cuda_stream != now.cuda_stream:
            self.ctx = torch.cuda.stream(stream)

    def __enter__(self):
        if self.ctx:
            self.ctx.__enter__()
        return self.handle

    def __exit__(self, *e):
        if self.ctx:
            self.ctx.__exit__(*e)


def _space(fn, *sizes):
    """(tensor, bytes) of the workspace a call needs."""
    need = ctypes.c_size_t()
    _check(fn(*sizes, ctypes.byref(need)))
    n = need.value
    return (torch.empty(n, dtype=torch.uint8, device="cuda") if n else None), n


# ------------------------------------------------------------------ embedding

def embed(tokens, table, scale=1.0, out=None, stream=None):
    """scale * table[tokens] (tq_embed): tokens int64 of any shape, table
    [V, D]; a token outside the table (-1: no shot) gives a row of zeros."""
    _typed(tokens, torch.int64, "tokens")
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    if table.dim() != 2:
        raise ValueError("table must be [V, D]")
    code = _type(table, "table")
    tp, V, D, ld = _rows(table, "table")
    V = table.shape[0]
    shape = tuple(tokens.shape) + (D,)
    with _On(stream) as s:
        if out is None:
            out = torch.empty(shape, dtype=table.dtype, device="cuda")
        op, _, _, ldo = _rows(out, "out", table.dtype, shape)
        _check(lib().tq_embed(tp, ld, code, V, D, tokens.data_ptr(), tokens.numel(), scale, op, ldo, s))
    return out


def embed_grad(tokens, grad_out, vocab, scale=1.0, grad=None, stream=None):
    """Gradient [vocab, D] of embed's table from that of its output
    (tq_embed_grad); bitwise reproducible."""
    _typed(tokens, torch.int64, "tokens")
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    if grad_out.dim() < 1 or tuple(grad_out.shape[:-1]) != tuple(tokens.shape):
        raise ValueError(f"grad_out must have shape {tuple(tokens.shape)} + [D], got {tuple(grad_out.shape)}")
    code = _type(grad_out, "grad_out")
    gp, _, D, ld = _rows(grad_out, "grad_out")
    N = tokens.numel()
    with _On(stream) as s:
        if grad is None:
            grad = torch.empty((vocab, D), dtype=grad_out.dtype, device="cuda")
        op, _, _, ldo = _rows(grad, "grad", grad_out.dtype, (vocab, D))
        ws, n = _space(lib().tq_embed_grad_workspace, vocab, D, N)
        _check(lib().tq_embed_grad(gp, ld, code, vocab, D, tokens.data_ptr(), N, scale, op, ldo, _ptr(ws), n, s))
    return grad


# ----------------------------------------------------------------- recurrence

def _scan_shape(x, g, lengths):
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError("x must be a [B, T, D] tensor")
    shape = tuple(x.shape)
    code = _type(x, "x")
    xs = _steps(x, "x", x.dtype, shape)
    gs = _steps(g, "g", x.dtype, shape)
    return code, shape, xs, gs, _dev(lengths, torch.int32, shape[:1], "lengths")


def gated_scan(x, g, h0=None, lengths=None, keep=False, y=None, h_last=None, states=None, stream=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(g_t) over the steps
    of x, g [B, T, D] (tq_gated_scan), from h0 float32 [B, D] (None: zeros);
    lengths int32 [B] (None: all T).  Returns (y, h_last), with keep=True
    (y, h_last, states), the states being what gated_scan_grad needs.  h_last
    may be the h0 tensor: the records' states then advance in place."""
    code, shape, xs, gs, lp = _scan_shape(x, g, lengths)
    B, T, D = shape
    hp = _dev(h0, torch.float32, (B, D), "h0")
    with _On(stream) as s:
        if y is None:
            y = torch.empty(shape, dtype=x.dtype, device="cuda")
        if h_last is None:
            h_last = torch.empty((B, D), dtype=torch.float32, device="cuda")
        pieces = -(-T // SCAN_PIECE)
        if states is None and keep:
            states = torch.empty((B, pieces, D), dtype=torch.float32, device="cuda")
        sp = _dev(states, torch.float32, (B, pieces, D), "states")
        ws, n = _space(lib().tq_gated_scan_workspace, B, T, D)
        _check(lib().tq_gated_scan(code, B, T, D, *xs, *gs, hp, lp, *_steps(y, "y", x.dtype, shape),
                                   _dev(h_last, torch.float32, (B, D), "h_last"), sp, _ptr(ws), n, s))
    return (y, h_last, states) if states is not None else (y, h_last)


def gated_scan_grad(x, g, states, dy, dh_last=None, lengths=None, dx=None, dg=None, dh0=None, stream=None):
    """(dx, dg, dh0) from the gradients of gated_scan's y and h_last (None:
    zeros) and the states it kept (tq_gated_scan_grad)."""
    code, shape, xs, gs, lp = _scan_shape(x, g, lengths)
    B, T, D = shape
    sp = _dev(states, torch.float32, (B, -(-T // SCAN_PIECE), D), "states")
    dp = _dev(dh_last, torch.float32, (B, D), "dh_last")
    dys = _steps(dy, "dy", x.dtype, shape)
    with _On(stream) as s:
        if dx is None:
            dx = torch.empty(shape, dtype=x.dtype, device="cuda")
        if dg is None:
            dg = torch.empty(shape, dtype=x.dtype, device="cuda")
        if dh0 is None:
            dh0 = torch.empty((B, D), dtype=torch.float32, device="cuda")
        ws, n = _space(lib().tq_gated_scan_workspace, B, T, D)
        _check(lib().tq_gated_scan_grad(code, B, T, D, *xs, *gs, sp, lp, *dys, dp, *_steps(dx, "dx", x.dtype, shape),
                                        *_steps(dg, "dg", x.dtype, shape), _dev(dh0, torch.float32, (B, D), "dh0"),
                                        _ptr(ws), n, s))
    return dx, dg, dh0


# ----------------------------------------------------------------- layer norm

def layer_norm(x, weight, bias=None, eps=1e-5, keep=False, y=None, stream=None):
    """Layer norm over the last axis of x (tq_layer_norm): y, or with keep=True
    (y, mean, rstd), the latter two float32 as layer_norm_grad needs them."""
    code = _type(x, "x")
    xp, N, D, ld = _rows(x, "x")
    wp = _dev(weight, x.dtype, (D,), "weight")
    bp = _dev(bias, x.dtype, (D,), "bias")
    with _On(stream) as s:
        if y is None:
            y = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        yp, _, _, ldy = _rows(y, "y", x.dtype, x.shape)
        mean = rstd = None
        if keep:
            mean, rstd = torch.empty((2,) + tuple(x.shape[:-1]), dtype=torch.float32, device="cuda")
        _check(lib().tq_layer_norm(xp, ld, code, N, D, wp, bp, eps, yp, ldy, _ptr(mean), _ptr(rstd), s))
    return (y, mean, rstd) if keep else y


def layer_norm_grad(x, weight, mean, rstd, dy, dx=None, stream=None):
    """(dx, dweight, dbias) of layer_norm (tq_layer_norm_grad)."""
    code = _type(x, "x")
    xp, N, D, ld = _rows(x, "x")
    wp = _dev(weight, x.dtype, (D,), "weight")
    mp = _dev(mean, torch.float32, x.shape[:-1], "mean")
    rp = _dev(rstd, torch.float32, x.shape[:-1], "rstd")
    dyp, _, _, ld_dy = _rows(dy, "dy", x.dtype, x.shape)
    with _On(stream) as s:
        if dx is None:
            dx = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        dxp, _, _, ld_dx = _rows(dx, "dx", x.dtype, x.shape)
        dw = torch.empty((D,), dtype=x.dtype, device="cuda")
        db = torch.empty((D,), dtype=x.dtype, device="cuda")
        ws, n = _space(lib().tq_layer_norm_grad_workspace, N, D)
        _check(lib().tq_layer_norm_grad(xp, ld, code, N, D, wp, mp, rp, dyp, ld_dy, dxp, ld_dx, dw.data_ptr(),
                                        db.data_ptr(), _ptr(ws), n, s))
    return dx, dw, db


# -------------------------------------------------------------- cross entropy

def _xent_args(hidden, weight, targets):
    code = _type(hidden, "hidden")
    hp, N, D, ldh = _rows(hidden, "hidden")
    if weight.dim() != 2 or weight.shape[1] != D:
        raise ValueError(f"weight must have shape [V, {D}], got {tuple(weight.shape)}")
    wp, _, _, ldw = _rows(weight, "weight", hidden.dtype)
    tp = _dev(targets, torch.int64, hidden.shape[:-1], "targets")
    return code, targets.numel(), weight.shape[0], D, hp, ldh, wp, ldw, tp


def softmax_xent(hidden, weight, targets, loss=None, lse=None, stream=None):
    """(loss, lse) float32, of the shape of targets, of the logits
    hidden @ weight^T (tq_softmax_xent); the loss of a target outside the
    vocabulary is 0."""
    code, N, V, D, hp, ldh, wp, ldw, tp = _xent_args(hidden, weight, targets)
    with _On(stream) as s:
        if loss is None:
            loss = torch.empty(targets.shape, dtype=torch.float32, device="cuda")
        if lse is None:
            lse = torch.empty(targets.shape, dtype=torch.float32, device="cuda")
        lp = _dev(loss, torch.float32, targets.shape, "loss")
        sp = _dev(lse, torch.float32, targets.shape, "lse")
        ws, n = _space(lib().tq_softmax_xent_workspace, code, N, V, D)
        _check(lib().tq_softmax_xent(hp, ldh, code, N, V, D, wp, ldw, tp, lp, sp, _ptr(ws), n, s))
    return loss, lse


def softmax_xent_grad(hidden, weight, targets, upstream, dhidden=None, dweight=None, stream=None):
    """(dhidden, dweight, loss, lse): the gradients of sum(upstream * loss) and
    softmax_xent's outputs, from one call (tq_softmax_xent_grad)."""
    code, N, V, D, hp, ldh, wp, ldw, tp = _xent_args(hidden, weight, targets)
    up = _dev(upstream, torch.float32, targets.shape, "upstream")
    with _On(stream) as s:
        if dhidden is None:
            dhidden = torch.empty(hidden.shape, dtype=hidden.dtype, device="cuda")
        if dweight is None:
            dweight = torch.empty(weight.shape, dtype=hidden.dtype, device="cuda")
        dhp, _, _, ld_dh = _rows(dhidden, "dhidden", hidden.dtype, hidden.shape)
        dwp, _, _, ld_dw = _rows(dweight, "dweight", hidden.dtype, weight.shape)
        loss = torch.empty(targets.shape, dtype=torch.float32, device="cuda")
        lse = torch.empty(targets.shape, dtype=torch.float32, device="cuda")
        ws, n = _space(lib().tq_softmax_xent_grad_workspace, code, N, V, D)
        _check(lib().tq_softmax_xent_grad(hp, ldh, code, N, V, D, wp, ldw, tp, up, dhp, ld_dh, dwp, ld_dw,
                                          loss.data_ptr(), lse.data_ptr(), _ptr(ws), n, s))
    return dhidden, dweight, loss, lse
