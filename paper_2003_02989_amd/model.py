"""Python binding of the operators of selective models of libtq
(include/tq_model.h): argument marshalling only.

Beside the sequence operators (seq.py), whose conventions hold here too: what a
selective model of measurement records runs over the steps of a record, how its
gradients are clipped and how a beam search answers with it.
Tensors live on the current HIP device; outputs and workspaces that the caller
does not give come from torch's allocator for the stream the call runs on.
"""
import collections
import ctypes
import math

import torch

from . import tq
from .seq import _TYPES, _call, _dense, _many, _on_stream, _ptr, _raw_stream, _rows, _space, _steps, _tensor, _typed

STATES_PIECE = 16  # TQ_STATES_PIECE: steps per state that selective_scan keeps for its gradient

_lib = None


def lib():
    """libtq.so with the prototypes of tq_model.h."""
    global _lib
    if _lib is None:
        L = tq.lib()
        vp, i32, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
        need = ctypes.POINTER(sz)
        steps = [vp, i64, i64]
        protos = {
            "tq_selective_scan_workspace": [i64, i64, i64, i64, need],
            "tq_selective_scan": [i32, i64, i64, i64, i64, *steps, *steps, vp, *steps, *steps, vp, *steps, vp, vp, vp,
                                  *steps, vp, vp, vp, sz, vp],
            "tq_selective_scan_grad_workspace": [i64, i64, i64, i64, need],
            "tq_selective_scan_grad": [i32, i64, i64, i64, i64, *steps, *steps, vp, *steps, *steps, vp, *steps, vp, vp, vp,
                                       *steps, vp, *steps, *steps, *steps, *steps, *steps, vp, vp, vp, vp, vp, sz, vp],
            "tq_causal_conv": [i32, i64, i64, i64, i64, *steps, vp, vp, vp, vp, i32, *steps, vp, vp],
            "tq_causal_conv_grad_workspace": [i64, i64, i64, i64, need],
            "tq_causal_conv_grad": [i32, i64, i64, i64, i64, *steps, vp, vp, vp, vp, i32, *steps, vp, *steps, vp, vp, vp, vp,
                                    sz, vp],
            "tq_clip_grad_norm_workspace": [i64, vp, need],
            "tq_clip_grad_norm": [i64, vp, vp, vp, f32, f32, vp, vp, vp, vp, sz, vp],
            "tq_beam_select_workspace": [i32, i64, i64, i64, i64, need],
            "tq_beam_select": [i32, i64, i64, i64, i64, vp, i64, vp, vp, ctypes.c_uint64, vp, vp, vp, vp, sz, vp],
            "tq_beam_reorder": [i64, vp, vp, vp, i64, i64, i64, vp, vp],
        }
        for name, args in protos.items():
            f = getattr(L, name)
            f.argtypes = args
            f.restype = ctypes.c_int
        _lib = L
    return _lib


_needs = {}


def _need(fn, *sizes):
    """Bytes of workspace that the library asks for with these sizes."""
    key = (fn,) + sizes
    n = _needs.get(key)
    if n is None:
        need = ctypes.c_size_t()
        _call(getattr(lib(), fn), *sizes, ctypes.byref(need))
        if len(_needs) > 4096:
            _needs.clear()
        n = _needs[key] = need.value
    return n


def _given_or_new(t, name, like):
    """A given output of the shape of `like` [B, T, N], or a new one, dense: (tensor,
    its steps)."""
    if t is not None:
        return t, _steps(t, name, like.dtype, like.shape)
    _, T, N = shape = like.shape
    t = like.new_empty(shape)
    return t, (t.data_ptr(), T * N, N)


def _floats(t, name, like, shape):
    """A given float32 output, or a new one, dense: (tensor, its pointer)."""
    if t is not None:
        return t, _dense(t, name, torch.float32, shape)
    t = torch.empty(shape, dtype=torch.float32, device=like.device)
    return t, t.data_ptr()


# ------------------------------------------------------------- selective scan

SelectiveGrads = collections.namedtuple("SelectiveGrads", "dx ddt dA dB dC dskip dz ddt_bias dh0")

_NONE = (None, 0, 0)


def _select_args(x, dt, A, B, C, skip, z, dt_bias, lengths):
    code, dev = _typed(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be a [B, T, D] tensor")
    shape, dtype = x.shape, x.dtype
    N, T, D = shape
    _tensor(A, "A", torch.float32)
    if A.dim() != 2 or A.shape[0] != D:
        raise ValueError(f"A must have shape [{D}, S], got {tuple(A.shape)}")
    S = A.shape[1]
    states = torch.Size((N, T, S))
    return dev, (code, N, T, D, S), (
        *_steps(x, "x", None, shape), *_steps(dt, "dt", dtype, shape), _dense(A, "A", torch.float32),
        *_steps(B, "B", dtype, states), *_steps(C, "C", dtype, states), _dense(skip, "skip", torch.float32, shape[2:]),
        *(_NONE if z is None else _steps(z, "z", dtype, shape)), _dense(dt_bias, "dt_bias", torch.float32, shape[2:])
    ), _dense(lengths, "lengths", torch.int32, shape[:1])


@_on_stream
def selective_scan(x, dt, A, B, C, skip=None, z=None, dt_bias=None, h0=None, lengths=None, keep=False, y=None,
                   h_last=None, states=None):
    """The selective state space scan (tq_selective_scan) over the steps of x, dt
    and z [B, T, D], B and C [B, T, S] with A float32 [D, S]: with
    d = softplus(dt + dt_bias), h_t = exp(d A) h_{t-1} + d x B_t from h0 float32
    [B, D, S], y_t = (C_t . h_t + skip x) silu(z).  None leaves skip, z, dt_bias
    out, starts from zeros, takes all T steps.  Returns (y, h_last), with
    keep=True (y, h_last, states), the states being what selective_scan_grad
    needs.  h_last may be the h0 tensor: the records' states then advance in place."""
    dev, sizes, args, lp = _select_args(x, dt, A, B, C, skip, z, dt_bias, lengths)
    _, N, T, D, S = sizes
    hp = _dense(h0, "h0", torch.float32, (N, D, S))
    y, ys = _given_or_new(y, "y", x)
    h_last, hlp = _floats(h_last, "h_last", x, (N, D, S))
    sp = None
    if keep or states is not None:
        states, sp = _floats(states, "states", x, (N, -(-T // STATES_PIECE), S, D))
    n = _need("tq_selective_scan_workspace", N, T, D, S)
    ws = _space(x, n)
    _call((_lib or lib()).tq_selective_scan, *sizes, *args, hp, lp, *ys, hlp, sp, _ptr(ws), n, _raw_stream(dev))
    return (y, h_last, states) if states is not None else (y, h_last)


@_on_stream
def selective_scan_grad(x, dt, A, B, C, states, dy, skip=None, z=None, dt_bias=None, dh_last=None, lengths=None,
                        dx=None, ddt=None, dB=None, dC=None, dz=None):
    """The gradients of selective_scan (tq_selective_scan_grad) from those of its
    y and h_last (None: zeros) and the states it kept: SelectiveGrads, with None for
    dz, dskip and ddt_bias where z, skip and dt_bias are None."""
    dev, sizes, args, lp = _select_args(x, dt, A, B, C, skip, z, dt_bias, lengths)
    _, N, T, D, S = sizes
    sp = _dense(states, "states", torch.float32, (N, -(-T // STATES_PIECE), S, D))
    dys = _steps(dy, "dy", x.dtype, x.shape)
    dhp = _dense(dh_last, "dh_last", torch.float32, (N, D, S))
    dx, dxs = _given_or_new(dx, "dx", x)
    ddt, ddts = _given_or_new(ddt, "ddt", x)
    dB, dBs = _given_or_new(dB, "dB", B)
    dC, dCs = _given_or_new(dC, "dC", C)
    if z is None:
        if dz is not None:
            raise ValueError("dz goes with z")
        dzs = _NONE
    else:
        dz, dzs = _given_or_new(dz, "dz", x)
    dA = torch.empty((D, S), dtype=torch.float32, device=x.device)
    dskip = None if skip is None else torch.empty((D,), dtype=torch.float32, device=x.device)
    dbias = None if dt_bias is None else torch.empty((D,), dtype=torch.float32, device=x.device)
    dh0 = torch.empty((N, D, S), dtype=torch.float32, device=x.device)
    n = _need("tq_selective_scan_grad_workspace", N, T, D, S)
    ws = _space(x, n)
    _call((_lib or lib()).tq_selective_scan_grad, *sizes, *args, sp, lp, *dys, dhp, *dxs, *ddts, *dzs, *dBs, *dCs,
          dA.data_ptr(), _ptr(dskip), _ptr(dbias), dh0.data_ptr(), _ptr(ws), n, _raw_stream(dev))
    if D == 0:  # sums over no channels, which the call leaves as they are
        dB.zero_()
        dC.zero_()
    return SelectiveGrads(dx, ddt, dA, dB, dC, dskip, dz, dbias, dh0)


# --------------------------------------------------------- causal convolution

def _conv_args(x, weight, bias, state, lengths, silu):
    code, dev = _typed(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be a [B, T, D] tensor")
    N, T, D = shape = x.shape
    dtype = x.dtype
    _tensor(weight, "weight", dtype)
    wp = _dense(weight, "weight", dtype)
    if weight.dim() != 2 or weight.shape[1] != D:
        raise ValueError(f"weight must have shape [K, {D}], got {tuple(weight.shape)}")
    K = weight.shape[0]
    return dev, (code, N, T, D, K), (*_steps(x, "x", None, shape), wp, _dense(bias, "bias", dtype, shape[2:]),
                                     _dense(state, "state", dtype, (N, K - 1, D)),
                                     _dense(lengths, "lengths", torch.int32, shape[:1]), bool(silu))


@_on_stream
def causal_conv(x, weight, bias=None, state=None, lengths=None, silu=True, y=None, last=None):
    """The causal convolution (tq_causal_conv) over the steps of x [B, T, D] with
    weight [K, D] and bias [D], followed by silu if wanted; state [B, K - 1, D]
    holds the inputs before the first step (None: zeros).  Returns (y, last), the
    latter the inputs before the next step; it may be the state tensor: records
    are then extended in place."""
    dev, sizes, args = _conv_args(x, weight, bias, state, lengths, silu)
    _, N, _, D, K = sizes
    y, ys = _given_or_new(y, "y", x)
    if last is None:
        last = x.new_empty((N, max(K - 1, 0), D))
        lp = last.data_ptr()
    else:
        lp = _dense(last, "last", x.dtype, (N, K - 1, D))
    _call((_lib or lib()).tq_causal_conv, *sizes, *args, *ys, lp, _raw_stream(dev))
    return y, last


ConvGrads = collections.namedtuple("ConvGrads", "dx dweight dbias dstate")


@_on_stream
def causal_conv_grad(x, weight, dy, bias=None, state=None, dlast=None, lengths=None, silu=True, dx=None):
    """The gradients of causal_conv (tq_causal_conv_grad) from those of its y and
    last (None: zeros): ConvGrads, with None for dbias and dstate where bias and
    state are None."""
    dev, sizes, args = _conv_args(x, weight, bias, state, lengths, silu)
    _, N, T, D, K = sizes
    dys = _steps(dy, "dy", x.dtype, x.shape)
    dp = _dense(dlast, "dlast", x.dtype, (N, K - 1, D))
    dx, dxs = _given_or_new(dx, "dx", x)
    dweight = torch.empty_like(weight)
    dbias = None if bias is None else torch.empty_like(bias)
    dstate = None if state is None else torch.empty_like(state)
    n = _need("tq_causal_conv_grad_workspace", N, T, D, K)
    ws = _space(x, n)
    _call((_lib or lib()).tq_causal_conv_grad, *sizes, *args, *dys, dp, *dxs, dweight.data_ptr(), _ptr(dbias),
          _ptr(dstate), _ptr(ws), n, _raw_stream(dev))
    return ConvGrads(dx, dweight, dbias, dstate)


# ----------------------------------------------------------- gradient clipping

def _list(kind, values):
    return (kind * len(values))(*values)


def _tensors(ts, name, like=None):
    """(pointers, type codes) of contiguous tensors, of the shapes of `like`."""
    ptrs, codes = [], []
    for t, k in zip(ts, ts if like is None else like):
        # (what _tensor and _dense check, without their calls where all is well)
        if _many or not isinstance(t, torch.Tensor) or not t.is_cuda or not t.is_contiguous() or t.shape != k.shape:
            _tensor(t, name, None, None if k is t else k.shape)
            _dense(t, name, None)
        code = _TYPES.get(t.dtype)
        if code is None:
            raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
        ptrs.append(t.data_ptr())
        codes.append(code)
    return ptrs, codes


def _apart(ptrs, ts, name):
    """Refuses outputs of which two are one."""
    if len(set(ptrs)) < len(ptrs):
        some = [p for p, t in zip(ptrs, ts) if t.numel()]
        if len(set(some)) < len(some):
            raise ValueError(f"{name} must be different tensors")


@_on_stream
def clip_grad_norm(grads, max_norm, scale=1.0, out=None):
    """(norm, outputs): the norm of all tensors of the list `grads` together, a
    float32 scalar on the device, times `scale`, and the tensors times scale, cut
    to max_norm where the norm is above it (tq_clip_grad_norm).  The outputs are
    the contiguous gradients themselves, each of them once, or the tensors of the
    list `out`, of their shapes and any of the types; none may be another one's
    gradient."""
    grads = list(grads)
    outs = grads if out is None else list(out)
    if len(outs) != len(grads):
        raise ValueError(f"out must be a list of {len(grads)} tensors, got {len(outs)}")
    if not grads:
        raise ValueError("grads must hold one tensor at least")
    n = len(grads)
    ptrs, codes = _tensors(grads, "grads")
    dev = grads[0].get_device()
    out_ptrs, out_codes = (ptrs, codes) if out is None else _tensors(outs, "out", grads)
    _apart(out_ptrs, outs, "grads" if out is None else "out")
    counts = _list(ctypes.c_int64, [t.numel() for t in grads])
    norm = torch.empty((), dtype=torch.float32, device=grads[0].device)
    need = ctypes.c_size_t()
    L = _lib or lib()
    _call(L.tq_clip_grad_norm_workspace, n, counts, ctypes.byref(need))
    ws = _space(norm, need.value)
    _call(L.tq_clip_grad_norm, n, _list(ctypes.c_void_p, ptrs), counts, _list(ctypes.c_int32, codes), max_norm, scale,
          _list(ctypes.c_void_p, out_ptrs), _list(ctypes.c_int32, out_codes), norm.data_ptr(), _ptr(ws), need.value,
          _raw_stream(dev))
    return norm, outs


# ----------------------------------------------------------------- beam search

@_on_stream
def beam_select(logits, scores, beams=None, last=None, end=-1):
    """One step of a beam search (tq_beam_select): the best `beams` (None: as many
    as there are) continuations of the beams of each record, from logits [R, W, V]
    and scores float32 [R, W].  last int64 [R, W], the beams' latest ids: those that
    are `end` go on as they are (None: no beam has ended).  Returns (scores float32,
    parents int32, tokens int64), each [R, beams], best first: beam `parents` goes
    on with id `tokens`."""
    code, dev = _typed(logits, "logits")
    if logits.dim() != 3:
        raise ValueError("logits must be a [R, W, V] tensor")
    zp, ld = _rows(logits, "logits")
    R, W, V = logits.shape
    K = W if beams is None else beams
    sp = _dense(scores, "scores", torch.float32, (R, W))
    lp = _dense(last, "last", torch.int64, (R, W))
    shape = (R, max(K, 0))
    best = torch.empty(shape, dtype=torch.float32, device=logits.device)
    parents = torch.empty(shape, dtype=torch.int32, device=logits.device)
    tokens = torch.empty(shape, dtype=torch.int64, device=logits.device)
    n = _need("tq_beam_select_workspace", code, R, W, V, K)
    ws = _space(logits, n)
    _call((_lib or lib()).tq_beam_select, code, R, W, V, K, zp, ld, sp, lp, end & 0xffffffffffffffff, best.data_ptr(),
          parents.data_ptr(), tokens.data_ptr(), _ptr(ws), n, _raw_stream(dev))
    return best, parents, tokens


@_on_stream
def beam_reorder(states, parents, out=None):
    """The states that go with beam_select's choice (tq_beam_reorder): for every
    tensor [R, W, ...] of the list `states`, of any type, the rows
    states[i][r, parents[r, k]] as a tensor [R, K, ...], new or that of the list
    `out`, which holds none of the states; zeros where a parent is not one of the W."""
    states = list(states)
    _tensor(parents, "parents", torch.int32)
    pp = _dense(parents, "parents", torch.int32)
    if parents.dim() != 2:
        raise ValueError("parents must be a [R, K] tensor")
    R, K = parents.shape
    for t in states:
        _tensor(t, "states")
        if t.dim() < 2 or t.shape[0] != R:
            raise ValueError(f"states must have shape [{R}, W, ...], got {tuple(t.shape)}")
        if t.shape[1] != states[0].shape[1]:
            raise ValueError("states must have one number of beams")
    if out is None:
        out = [t.new_empty((R, K) + t.shape[2:]) for t in states]
    out = list(out)
    if len(out) != len(states):
        raise ValueError(f"out must be a list of {len(states)} tensors, got {len(out)}")
    if not states:
        return out
    W = states[0].shape[1]
    ins, outs, rows = [], [], []
    for t, o in zip(states, out):
        row = t.shape[2:]
        ins.append(_dense(t, "states", None))
        outs.append(_dense(o, "out", t.dtype, (R, K) + row))
        rows.append(math.prod(row) * t.element_size())
    _apart(outs, out, "out")
    _call((_lib or lib()).tq_beam_reorder, len(states), _list(ctypes.c_void_p, ins), _list(ctypes.c_void_p, outs),
          _list(ctypes.c_int64, rows), R, W, K, pp, _raw_stream(parents.get_device()))
    return out
