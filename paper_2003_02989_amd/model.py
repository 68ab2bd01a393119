"""Python binding of the operators of selective models of libtq
(include/tq_model.h): argument marshalling only.

Beside the sequence operators (seq.py), whose conventions hold here too: what a
selective model of measurement records runs over the steps of a record.
Tensors live on the current HIP device; outputs and workspaces that the caller
does not give come from torch's allocator for the stream the call runs on.
"""
import collections
import ctypes

import torch

from . import tq
from .seq import _call, _dense, _on_stream, _ptr, _raw_stream, _space, _steps, _steps_out, _tensor, _typed

STATES_PIECE = 16  # TQ_STATES_PIECE: steps per state that selective_scan keeps for its gradient

_lib = None


def lib():
    """libtq.so with the prototypes of tq_model.h."""
    global _lib
    if _lib is None:
        L = tq.lib()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
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
    y, ys = _steps_out(y, "y", x)
    if h_last is None:
        h_last = torch.empty((N, D, S), dtype=torch.float32, device=x.device)
    pieces = -(-T // STATES_PIECE)
    if states is None and keep:
        states = torch.empty((N, pieces, S, D), dtype=torch.float32, device=x.device)
    n = _need("tq_selective_scan_workspace", N, T, D, S)
    ws = _space(x, n)
    _call((_lib or lib()).tq_selective_scan, *sizes, *args, hp, lp, *ys,
          _dense(h_last, "h_last", torch.float32, (N, D, S)),
          _dense(states, "states", torch.float32, (N, pieces, S, D)), _ptr(ws), n, _raw_stream(dev))
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
    dx, dxs = _steps_out(dx, "dx", x)
    ddt, ddts = _steps_out(ddt, "ddt", x)
    dB, dBs = _steps_out(dB, "dB", B)
    dC, dCs = _steps_out(dC, "dC", C)
    if z is None:
        if dz is not None:
            raise ValueError("dz goes with z")
        dzs = _NONE
    else:
        dz, dzs = _steps_out(dz, "dz", x)
    dA = torch.empty((D, S), dtype=torch.float32, device=x.device)
    dskip = None if skip is None else torch.empty((D,), dtype=torch.float32, device=x.device)
    dbias = None if dt_bias is None else torch.empty((D,), dtype=torch.float32, device=x.device)
    dh0 = torch.empty((N, D, S), dtype=torch.float32, device=x.device)
    n = _need("tq_selective_scan_grad_workspace", N, T, D, S)
    ws = _space(x, n)
    _call((_lib or lib()).tq_selective_scan_grad, *sizes, *args, sp, lp, *dys, dhp, *dxs, *ddts, *dzs, *dBs, *dCs,
          dA.data_ptr(), _ptr(dskip), _ptr(dbias), dh0.data_ptr(), _ptr(ws), n, _raw_stream(dev))
    return SelectiveGrads(dx, ddt, dA, dB, dC, dskip, dz, dbias, dh0)


# --------------------------------------------------------- causal convolution

def _conv_args(x, weight, bias, state, lengths, silu):
    code, dev = _typed(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be a [B, T, D] tensor")
    N, T, D = shape = x.shape
    dtype = x.dtype
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
    y, ys = _steps_out(y, "y", x)
    if last is None:
        last = x.new_empty((N, max(K - 1, 0), D))
    _call((_lib or lib()).tq_causal_conv, *sizes, *args, *ys, _dense(last, "last", x.dtype, (N, K - 1, D)),
          _raw_stream(dev))
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
    dx, dxs = _steps_out(dx, "dx", x)
    dweight = torch.empty_like(weight)
    dbias = None if bias is None else torch.empty_like(bias)
    dstate = None if state is None else torch.empty_like(state)
    n = _need("tq_causal_conv_grad_workspace", N, T, D, K)
    ws = _space(x, n)
    _call((_lib or lib()).tq_causal_conv_grad, *sizes, *args, *dys, dp, *dxs, dweight.data_ptr(), _ptr(dbias),
          _ptr(dstate), _ptr(ws), n, _raw_stream(dev))
    return ConvGrads(dx, dweight, dbias, dstate)
