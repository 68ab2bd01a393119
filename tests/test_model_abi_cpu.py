"""Host-side checks of tq_model.h, no GPU needed: every declared function is
exported, and arguments that do not fit are refused before any device call."""
import ctypes
import os
import re

import pytest
import torch

from paper_2003_02989_amd import model, tq
from test_seq_abi_cpu import BF16, F16, F32, P, changed, refused, space

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "tq_model.h")).read()
    names = sorted(set(re.findall(r"^tq_status (tq_[a-z_]+)\(", text, re.M)))
    assert len(names) == 12
    for n in names:
        assert hasattr(model.lib(), n), n
    assert int(re.search(r"#define TQ_STATES_PIECE (\d+)", text).group(1)) == model.STATES_PIECE


def test_selective_scan_refusals():
    L = model.lib()
    B, T, D, S = 2, 5000, 8, 4
    need = space(L.tq_selective_scan_workspace, B, T, D, S)
    assert need > 0 and space(L.tq_selective_scan_workspace, B, 10, D, S) == 0
    st, ss = [T * D, D], [T * S, S]
    ok = [F32, B, T, D, S, P, *st, P, *st, P, P, *ss, P, *ss, P, P, *st, P, P, P, P, *st, P, P, P, need, None]
    x, dt, A, Bm, Cm, skip, z, bias, h0, n, y, h, states, ws = 5, 8, 11, 12, 15, 18, 19, 22, 23, 24, 25, 28, 29, 30
    for k, v in ((0, 5), (1, -1), (2, -1), (3, -1), (4, 0), (4, -1), (x, None), (x + 1, -1), (dt, None), (A, None),
                 (A, P + 2), (Bm, None), (Bm + 2, -4), (Cm, None), (skip, P + 1), (z, P + 2), (z + 1, -1), (bias, P + 2),
                 (h0, P + 1), (n, P + 2), (y, None), (y + 1, D), (y + 2, D - 1), (h, P + 2), (states, P + 1), (ws, None),
                 (ws, P + 8), (ws + 1, need - 1)):
        refused(tq.TQ_E_INVALID, L.tq_selective_scan, *changed(ok, k, v))
    for sizes in ((2, T, D, 65), (2, T, (1 << 20) + 1, S), (1 << 20, 1 << 20, 64, S), (1 << 31, 1, 1, 1),
                  ((1 << 31) - 1, 0, 65, 1)):
        refused(tq.TQ_E_UNSUPPORTED, L.tq_selective_scan, F32, *sizes, *ok[5:])
        refused(tq.TQ_E_UNSUPPORTED, L.tq_selective_scan_workspace, *sizes, ctypes.byref(ctypes.c_size_t()))
        refused(tq.TQ_E_UNSUPPORTED, L.tq_selective_scan_grad_workspace, *sizes, ctypes.byref(ctypes.c_size_t()))
    refused(tq.TQ_E_INVALID, L.tq_selective_scan_workspace, B, T, D, S, None)
    assert L.tq_selective_scan(*changed(ok, 1, 0)) == tq.TQ_OK  # nothing to do
    assert L.tq_selective_scan(*changed(ok, 3, 0)) == tq.TQ_OK


def test_selective_scan_grad_refusals():
    L = model.lib()
    B, T, D, S = 2, 50, 8, 4
    need = space(L.tq_selective_scan_grad_workspace, B, T, D, S)
    st, ss = [T * D, D], [T * S, S]
    ok = [BF16, B, T, D, S, P, *st, P, *st, P, P, *ss, P, *ss, P, P, *st, P, P, P, P, *st, P, P, *st, P, *st, P, *st, P, *ss,
          P, *ss, P, P, P, P, P, need, None]
    states, dy, dh, dx, ddt, dz, dB, dC, dA, ws = 23, 25, 28, 29, 32, 35, 38, 41, 44, 48
    assert ok[ws + 1] == need
    for k, v in ((0, 5), (1, -1), (4, 0), (5, None), (8, None), (11, None), (12, None), (15, None), (18, P + 2), (22, P + 1),
                 (states, None), (states, P + 2), (dy, None), (dy, P + 1), (dh, P + 2), (dx, None), (dx + 2, D - 1),
                 (ddt, None), (ddt + 1, D), (dz, None), (dz + 2, 1), (dB, None), (dB + 2, S - 1), (dC, None), (dC + 1, S),
                 (dA, None), (dA + 1, P + 2), (dA + 2, P + 2), (dA + 3, P + 2), (ws, None), (ws, P + 128),
                 (ws + 1, need - 1), (19, None)):
        refused(tq.TQ_E_INVALID, L.tq_selective_scan_grad, *changed(ok, k, v))
    refused(tq.TQ_E_UNSUPPORTED, L.tq_selective_scan_grad, *changed(ok, 4, 65))
    assert L.tq_selective_scan_grad(*changed(ok, 3, 0)) == tq.TQ_OK


def test_causal_conv_refusals():
    L = model.lib()
    B, T, D, K = 3, 40, 8, 4
    st = [T * D, D]
    ok = [F16, B, T, D, K, P, *st, P, P, P, P, 1, P, *st, P, None]
    for k, v in ((0, 3), (1, -1), (2, -1), (3, -1), (4, 0), (5, None), (6, -1), (8, None), (9, P + 1), (10, P + 1),
                 (11, P + 2), (13, None), (13, P + 1), (14, D), (15, D - 1), (16, P + 1)):
        refused(tq.TQ_E_INVALID, L.tq_causal_conv, *changed(ok, k, v))
    for sizes in ((B, T, D, 9), (B, T, (1 << 20) + 1, K), (1 << 30, 16, 8, K), (1 << 30, 8, 7, K), (1 << 20, 0, 1 << 20, K)):
        refused(tq.TQ_E_UNSUPPORTED, L.tq_causal_conv, F16, *sizes, *ok[5:])
        refused(tq.TQ_E_UNSUPPORTED, L.tq_causal_conv_grad_workspace, *sizes, ctypes.byref(ctypes.c_size_t()))
    assert L.tq_causal_conv(*changed(ok, 1, 0)) == tq.TQ_OK
    need = space(L.tq_causal_conv_grad_workspace, B, T, D, K)
    gk = [F16, B, T, D, K, P, *st, P, P, P, P, 1, P, *st, P, P, *st, P, P, P, P, need, None]
    for k, v in ((0, 3), (4, 0), (5, None), (8, None), (13, None), (14, -1), (16, P + 1), (17, None), (18, D), (20, None),
                 (21, P + 1), (22, P + 1), (23, None), (23, P + 64), (24, need - 1)):
        refused(tq.TQ_E_INVALID, L.tq_causal_conv_grad, *changed(gk, k, v))
    assert L.tq_causal_conv_grad(*changed(gk, 3, 0)) == tq.TQ_OK


def lists(*values):
    kinds = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32)
    return [None if v is None else (k * len(v))(*v) for k, v in zip(kinds, values)]


def test_clip_grad_norm_refusals():
    L = model.lib()

    def call(grads=(P, 2 * P), counts=(100000, 5), types=(F16, F32), outs=(3 * P, 4 * P), out_types=(F32, F32), n=2, most=1.0,
             scale=1.0, norm=P, ws=P, need=None):
        g, c, t, o, ot = lists(grads, counts, types, outs, out_types)
        if need is None:
            need = space(L.tq_clip_grad_norm_workspace, 2, (ctypes.c_int64 * 2)(100000, 5))
        return L.tq_clip_grad_norm(n, g, c, t, most, scale, o, ot, norm, ws, need, None)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(n=-1), dict(counts=None), dict(counts=(-1, 5)), dict(grads=None), dict(types=None), dict(outs=None),
                dict(out_types=None), dict(types=(3, F32)), dict(out_types=(F32, -1)), dict(grads=(None, P)),
                dict(grads=(P + 1, P)), dict(grads=(P, P + 2)), dict(outs=(P + 2, P)), dict(outs=(3 * P, None)), dict(most=-1.0),
                dict(most=nan), dict(scale=0.0), dict(scale=-1.0), dict(scale=inf), dict(scale=nan), dict(norm=None),
                dict(norm=P + 2), dict(ws=None), dict(ws=P + 64), dict(need=8), dict(outs=(P, 2 * P))):
        assert call(**bad) == tq.TQ_E_INVALID, bad
        assert tq.lib().tq_last_error()
    assert call(n=1 << 20) == tq.TQ_E_UNSUPPORTED
    assert call(counts=(1 << 40, 5)) == tq.TQ_E_UNSUPPORTED
    assert space(L.tq_clip_grad_norm_workspace, 2, (ctypes.c_int64 * 2)(100, 5)) == 0
    refused(tq.TQ_E_INVALID, L.tq_clip_grad_norm_workspace, 2, (ctypes.c_int64 * 2)(100, 5), None)


def test_beam_select_refusals():
    L = model.lib()
    R, W, V, K = 3, 4, 100000, 5
    need = space(L.tq_beam_select_workspace, BF16, R, W, V, K)
    assert need > 0 and space(L.tq_beam_select_workspace, F32, R, W, 100, K) == 0
    ok = [BF16, R, W, V, K, P, V, P, P, 7, P, P, P, P, need, None]
    for k, v in ((0, 3), (1, -1), (2, 0), (3, 0), (3, -1), (4, 0), (5, None), (5, P + 1), (6, V - 1), (7, None), (7, P + 2),
                 (8, P + 4), (9, V), (9, (1 << 64) - 1), (10, None), (11, None), (11, P + 2), (12, None), (12, P + 4),
                 (13, None), (13, P + 8), (14, need - 1)):
        refused(tq.TQ_E_INVALID, L.tq_beam_select, *changed(ok, k, v))
    refused(tq.TQ_E_INVALID, L.tq_beam_select, *changed(changed(ok, 3, 1), 4, 5))  # 4 candidates
    for k, v in ((2, 65), (4, 65), (3, 1 << 31), (1, 1 << 31), (1, 1 << 29)):
        refused(tq.TQ_E_UNSUPPORTED, L.tq_beam_select, *changed(ok, k, v))
    assert L.tq_beam_select(*changed(ok, 1, 0)) == tq.TQ_OK


def test_beam_reorder_refusals():
    L = model.lib()

    def call(ins=(P, 2 * P), outs=(3 * P, 4 * P), rows=(16, 3), R=2, W=3, K=3, n=2, parents=P):
        i, r, _, o, _ = lists(ins, rows, (0, 0), outs, (0, 0))
        return L.tq_beam_reorder(n, i, o, r, R, W, K, parents, None)
    for bad in (dict(n=-1), dict(ins=None), dict(outs=None), dict(rows=None), dict(rows=(-1, 3)), dict(R=-1), dict(W=-1),
                dict(K=-1), dict(ins=(None, P)), dict(outs=(P, 4 * P)), dict(outs=(3 * P, None)), dict(parents=None),
                dict(parents=P + 2)):
        assert call(**bad) == tq.TQ_E_INVALID, bad
    for bad in (dict(n=1 << 20), dict(rows=(1 << 40, 3)), dict(R=1 << 31), dict(R=1 << 20, K=1 << 12),
                dict(R=1 << 30, K=1, rows=(1 << 30, 3))):
        assert call(**bad) == tq.TQ_E_UNSUPPORTED, bad
    for nothing in (dict(n=0), dict(R=0), dict(K=0)):
        assert call(**nothing) == tq.TQ_OK


def test_binding_refuses_host_tensors():
    x, w = torch.zeros((2, 3, 4)), torch.zeros((4, 4))
    s = torch.zeros((2, 3, 5))
    A = torch.zeros((4, 5))
    for call in (lambda: model.selective_scan(x, x, A, s, s), lambda: model.selective_scan_grad(x, x, A, s, s, A, x),
                 lambda: model.causal_conv(x, w), lambda: model.causal_conv_grad(x, w, x),
                 lambda: model.clip_grad_norm([x], 1.0), lambda: model.beam_select(x, x[..., 0]),
                 lambda: model.beam_reorder([x], torch.zeros((2, 3), dtype=torch.int32))):
        with pytest.raises(TypeError):
            call()
