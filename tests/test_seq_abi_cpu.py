"""Host-side checks of tq_seq.h, no GPU needed: every declared function is
exported, and arguments that do not fit are refused before any device call."""
import ctypes
import os
import re

import pytest

from paper_2003_02989_amd import seq, tq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # stands for a device pointer: refused calls never look behind it
F32, BF16, F16 = 0, 1, 2


def test_every_declared_symbol_is_exported():
    text = open(os.path.join(ROOT, "include", "tq_seq.h")).read()
    names = sorted(set(re.findall(r"^tq_status (tq_[a-z_]+)\(", text, re.M)))
    assert len(names) == 13
    for n in names:
        assert hasattr(seq.lib(), n), n
    assert int(re.search(r"#define TQ_SCAN_PIECE (\d+)", text).group(1)) == seq.SCAN_PIECE


def space(fn, *sizes):
    n = ctypes.c_size_t()
    assert fn(*sizes, ctypes.byref(n)) == tq.TQ_OK, tq.lib().tq_last_error()
    return n.value


def refused(status, fn, *args):
    assert fn(*args) == status
    assert tq.lib().tq_last_error()


def changed(args, k, v):
    return args[:k] + [v] + args[k + 1:]


def test_embed_refusals():
    f = seq.lib().tq_embed
    ok = [P, 8, F32, 5, 8, P, 3, 1.0, P, 8, None]
    for k, v in ((0, None), (1, 7), (2, 3), (2, -1), (3, -1), (4, -1), (5, None), (6, -1), (8, None), (9, 7), (0, P + 2),
                 (5, P + 4), (8, P + 1)):
        refused(tq.TQ_E_INVALID, f, *changed(ok, k, v))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(ok, 3, 1 << 31))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(ok, 6, 1 << 31))
    assert f(*changed(ok, 6, 0)) == tq.TQ_OK  # nothing to do


def test_embed_grad_refusals():
    f = seq.lib().tq_embed_grad
    need = space(seq.lib().tq_embed_grad_workspace, 5, 8, 3000)
    assert need > 0 and space(seq.lib().tq_embed_grad_workspace, 5, 8, 3) == 0
    ok = [P, 8, BF16, 5, 8, P, 3000, 1.0, P, 8, P, need, None]
    for k, v in ((0, None), (1, 7), (2, 9), (3, -1), (5, None), (8, None), (9, 7), (10, None), (10, P + 16),
                 (11, need - 1), (0, P + 1)):
        refused(tq.TQ_E_INVALID, f, *changed(ok, k, v))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(ok, 4, (1 << 20) + 1))
    refused(tq.TQ_E_INVALID, seq.lib().tq_embed_grad_workspace, 5, 8, 3, None)
    assert f(*changed(ok, 3, 0)) == tq.TQ_OK


def test_gated_scan_refusals():
    f, g = seq.lib().tq_gated_scan, seq.lib().tq_gated_scan_grad
    B, T, D = 2, 1000, 8
    need = space(seq.lib().tq_gated_scan_workspace, B, T, D)
    assert need > 0
    st = [T * D, D]
    ok = [F32, B, T, D, P, *st, P, *st, P, None, P, *st, P, None, P, need, None]
    for k, v in ((0, 5), (1, -1), (2, -1), (3, -1), (4, None), (5, -1), (7, None), (9, -8), (12, None), (12, P + 2),
                 (13, D), (14, D - 1), (10, P + 1), (15, P + 2), (17, None), (17, P + 8), (18, need - 1)):
        refused(tq.TQ_E_INVALID, f, *changed(ok, k, v))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(ok, 2, 1 << 31))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(changed(ok, 1, 1 << 30), 3, 1 << 20))
    assert f(*changed(ok, 1, 0)) == tq.TQ_OK
    gk = [F32, B, T, D, P, *st, P, *st, P, None, P, *st, None, P, *st, P, *st, None, P, need, None]
    for k, v in ((0, 5), (4, None), (7, None), (10, None), (12, None), (16, None), (17, D), (19, None), (21, D - 1),
                 (23, None), (24, need - 1)):
        refused(tq.TQ_E_INVALID, g, *changed(gk, k, v))
    # steps outermost is a layout like any other
    refused(tq.TQ_E_INVALID, f, *changed(changed(changed(ok, 13, D), 14, 2 * D), 18, 0))
    assert b"workspace" in tq.lib().tq_last_error()


def test_layer_norm_refusals():
    f, g = seq.lib().tq_layer_norm, seq.lib().tq_layer_norm_grad
    ok = [P, 8, F16, 4, 8, P, P, 1e-5, P, 8, P, P, None]
    for k, v in ((0, None), (1, 7), (2, 4), (3, -1), (5, None), (7, -1.0), (7, float("nan")), (8, None), (9, 7),
                 (10, None), (11, None), (6, P + 1)):
        refused(tq.TQ_E_INVALID, f, *changed(ok, k, v))
    assert f(*changed(ok, 3, 0)) == tq.TQ_OK
    need = space(seq.lib().tq_layer_norm_grad_workspace, 4, 8)
    gk = [P, 8, F16, 4, 8, P, P, P, P, 8, P, 8, P, P, P, need, None]
    for k, v in ((0, None), (1, 7), (5, None), (6, None), (7, None), (8, None), (9, 7), (10, None), (11, 7), (12, None),
                 (13, P + 1), (14, None), (15, need - 1)):
        refused(tq.TQ_E_INVALID, g, *changed(gk, k, v))


def test_softmax_xent_refusals():
    f, g = seq.lib().tq_softmax_xent, seq.lib().tq_softmax_xent_grad
    need = space(seq.lib().tq_softmax_xent_workspace, BF16, 100, 7, 8)
    ok = [P, 8, BF16, 100, 7, 8, P, 8, P, P, P, P, need, None]
    for k, v in ((0, None), (1, 7), (2, 3), (3, -1), (4, 0), (4, -1), (6, None), (7, 7), (8, None), (9, None),
                 (10, None), (11, None), (12, need - 1), (0, P + 1), (8, P + 4)):
        refused(tq.TQ_E_INVALID, f, *changed(ok, k, v))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(changed(ok, 3, 1 << 30), 4, 1 << 30))
    refused(tq.TQ_E_UNSUPPORTED, f, *changed(changed(changed(ok, 5, 1 << 21), 1, 1 << 21), 7, 1 << 21))
    assert f(*changed(ok, 3, 0)) == tq.TQ_OK
    need = space(seq.lib().tq_softmax_xent_grad_workspace, F32, 100, 7, 8)
    gk = [P, 8, F32, 100, 7, 8, P, 8, P, P, P, 8, P, 8, P, P, P, need, None]
    for k, v in ((0, None), (1, 7), (6, None), (7, 7), (8, None), (9, None), (10, None), (11, 7), (12, None), (13, 7),
                 (14, None), (15, None), (16, None), (16, P + 128), (17, need - 1)):
        refused(tq.TQ_E_INVALID, g, *changed(gk, k, v))
    # empty sizes ask for workspaces without failing
    for sizes in ((F32, 0, 7, 8), (BF16, 100, 7, 0), (F16, 0, 7, 0), (F32, 1, 1, 1)):
        space(seq.lib().tq_softmax_xent_grad_workspace, *sizes)
        space(seq.lib().tq_softmax_xent_workspace, *sizes)


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((3, 4))
    t = torch.zeros(3, dtype=torch.int64)
    for call in (lambda: seq.embed(t, x), lambda: seq.embed_grad(t, x, 5), lambda: seq.layer_norm(x, x[0]),
                 lambda: seq.gated_scan(x[None], x[None]), lambda: seq.softmax_xent(x, x, t)):
        with pytest.raises(TypeError):
            call()
