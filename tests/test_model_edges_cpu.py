"""Calls of the operators of selective models at the ends of what the header
allows, without a GPU."""
import pytest
import torch

import launches as la
from paper_2003_02989_amd import model, seq
from test_model_binding_cpu import fake
from test_model_launches_cpu import _lists, run  # noqa: F401 (the fixture serves here too)

P, ALL = la.P, la.ALL


@pytest.mark.parametrize("given", [False, True])
def test_no_channels_still_give_gradients_of_b_and_c(monkeypatch, given):
    """dB and dC are sums over the channels: of none, zeros."""
    called = []
    monkeypatch.setattr(model, "_call", lambda f, *a: called.append(f.__name__))
    monkeypatch.setattr(model, "_raw_stream", lambda dev: None)
    monkeypatch.setattr(model, "_space", lambda like, n: None)
    x, s, A = fake(2, 40, 0), fake(2, 40, 5), fake(0, 5)
    out = {}
    if given:  # views of one array, whose other columns stay
        room = fake(2, 40, 12).fill_(float("nan"))
        out = dict(dB=room[..., :5], dC=room[..., 5:10])
    else:  # what the memory held
        new = torch.Tensor.new_empty
        monkeypatch.setattr(torch.Tensor, "new_empty", lambda t, shape: new(t, shape).fill_(float("nan")))
    g = model.selective_scan_grad(x, x, A, s, s, fake(2, 3, 5, 0), x, **out)
    assert called[-1] == "tq_selective_scan_grad"
    for got in (g.dB, g.dC):
        assert got.shape == (2, 40, 5) and bool((got == 0).all())
    assert not given or (g.dB is out["dB"] and bool(torch.isnan(room[..., 10:]).all()))


def clip(grads, outs, counts):
    n = len(grads)
    return ("tq_clip_grad_norm", n, grads, counts, [0] * n, 1.0, 1.0, outs, [0] * n, P, P, ALL, None)


def test_clipping_refuses_outputs_that_are_other_gradients(tmp_path):
    """One workgroup would read what another has written."""
    a, b, c = P, 2 * P, 3 * P
    good = [clip([a, b], [a, b], [9, 9]), clip([a, b, c], [a, 4 * P, c], [9, 70000, 9]), clip([a, a], [b, c], [9, 9]),
            clip([a, a], [a, a], [9, 0]), clip([a, b], [b, a], [0, 9]), clip([a, None, b], [b, None, 4 * P], [9, 0, 0])]
    run(good, tmp_path)
    bad = [clip([a, b], [b, c], [9, 9]), clip([a, b], [b, a], [9, 9]), clip([a, a], [a, a], [9, 9]),
           clip([a, b, a], [a, b, c], [9, 9, 9]), clip([a, b, c], [4 * P, 5 * P, a], [9, 70000, 9])]
    assert all(g["rc"] == 1 and not g["kernels"] for g in la.recorded(bad, tmp_path)[0])


def test_clipping_refuses_a_tensor_twice(monkeypatch):
    monkeypatch.setattr(model, "_call", lambda f, *a: None)
    monkeypatch.setattr(model, "_raw_stream", lambda dev: None)
    x, y, o, none = fake(3, 4), fake(3, 4), fake(3, 4), fake(0)
    model.clip_grad_norm([x, y, none, none], 1.0)
    model.clip_grad_norm([x, x], 1.0, out=[o, y])
    for grads, out in (([x, x], None), ([x, y], [o, o]), ([x, y, none], [o, o, none])):
        with pytest.raises(ValueError):
            model.clip_grad_norm(grads, 1.0, out=out)


def reorder(ins, outs, rows, R=2, W=3, K=3):
    return ("tq_beam_reorder", len(ins), ins, outs, rows, R, W, K, P, None)


def test_reordering_refuses_outputs_that_are_states(tmp_path):
    a, b, c = P, 2 * P, 3 * P
    run([reorder([a, a], [b, c], [8, 8]), reorder([a, b], [c, a], [8, 0]), reorder([a, b], [c, a], [0, 8]),
         reorder([None, None], [a, b], [8, 8], W=0)], tmp_path)
    bad = [reorder([a, b], [c, a], [8, 8]), reorder([a, b], [b, a], [8, 8]), reorder([a, b, 4 * P], [c, 5 * P, b], [1, 9000, 5])]
    assert all(g["rc"] == 1 and not g["kernels"] for g in la.recorded(bad, tmp_path)[0])


def test_reordering_refuses_an_output_twice(monkeypatch):
    monkeypatch.setattr(model, "_call", lambda f, *a: None)
    monkeypatch.setattr(model, "_raw_stream", lambda dev: None)
    x, y, o, p = fake(2, 3, 4), fake(2, 3, 4), fake(2, 5, 4), fake(2, 5, dtype=torch.int32)
    none, gone = fake(2, 3, 0), fake(2, 5, 0)
    model.beam_reorder([x, x], p)
    model.beam_reorder([x, none, none], p, out=[o, gone, gone])
    model.beam_reorder([x[:0], y[:0]], p[:0], out=[o[:0], o[:0]])
    with pytest.raises(ValueError):
        model.beam_reorder([x, y], p, out=[o, o])


def test_arrays_of_no_elements_may_have_any_strides():
    """Views of every second column, as a table's without steps or records are."""
    for shape in ((2, 0, 8), (0, 3, 8)):
        t = fake(*shape)[..., ::2]
        assert seq._steps(t, "x", None, t.shape)[1:] == t.stride()[:2]
    with pytest.raises(ValueError):
        seq._steps(fake(2, 3, 8)[..., ::2], "x", None, (2, 3, 4))
