"""The model binding's own argument checks, without a GPU: what does not fit is
refused before the library is called."""
import pytest
import torch

from paper_2003_02989_amd import model, seq


class Fake(torch.Tensor):  # stands for a device tensor
    is_cuda = True

    def get_device(self):
        return 0


def fake(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(Fake)


@pytest.fixture(autouse=True)
def _no_library(monkeypatch):
    call = seq._call

    def called(f, *a):
        assert f.__name__.endswith("_workspace"), "the library was called"
        call(f, *a)
    monkeypatch.setattr(model, "_call", called)


def refuse(error, f, *args, **kw):
    with pytest.raises(error):
        f(*args, **kw)


def test_selective_scan_shapes_and_types():
    x, s, A = fake(2, 3, 4), fake(2, 3, 5), fake(4, 5)
    half = fake(2, 3, 4, dtype=torch.float16)
    ok = dict(x=x, dt=x, A=A, B=s, C=s)
    for name, bad in (("x", fake(3, 4)), ("dt", fake(2, 3, 5)), ("A", fake(5, 5)), ("A", fake(4)), ("B", fake(2, 3, 4)),
                      ("C", fake(2, 2, 5)), ("skip", fake(5)), ("z", fake(2, 3, 1)), ("dt_bias", fake(1, 4)),
                      ("h0", fake(2, 5, 4)), ("lengths", fake(3, dtype=torch.int32)), ("y", fake(2, 3, 5)),
                      ("h_last", fake(2, 4, 4)), ("states", fake(2, 2, 5, 4))):
        refuse(ValueError, model.selective_scan, **{**ok, "h_last": fake(2, 4, 5), name: bad})
    for name, bad in (("x", fake(2, 3, 4, dtype=torch.float64)), ("dt", half), ("z", half), ("A", half[0]),
                      ("skip", fake(4, dtype=torch.float16)), ("lengths", fake(2, dtype=torch.int64)),
                      ("h0", fake(2, 4, 5, dtype=torch.bfloat16))):
        refuse(TypeError, model.selective_scan, **{**ok, name: bad})
    refuse(ValueError, model.selective_scan, **{**ok, "dt": fake(2, 3, 8)[..., ::2]})
    refuse(ValueError, model.selective_scan, **{**ok, "A": fake(5, 4).t()})
    states = fake(2, 1, 5, 4)
    refuse(ValueError, model.selective_scan_grad, **ok, states=fake(2, 1, 4, 5), dy=x)
    refuse(ValueError, model.selective_scan_grad, **ok, states=states, dy=fake(2, 3, 3))
    refuse(TypeError, model.selective_scan_grad, **ok, states=states, dy=half)
    refuse(ValueError, model.selective_scan_grad, **ok, states=states, dy=x, dz=x)
    refuse(ValueError, model.selective_scan_grad, **ok, states=states, dy=x, dB=x)


def test_causal_conv_shapes_and_types():
    x, w = fake(2, 3, 4), fake(4, 4)
    for kw in (dict(weight=fake(4, 5)), dict(weight=fake(4)), dict(bias=fake(5)), dict(state=fake(2, 4, 4)),
               dict(lengths=fake(3, dtype=torch.int32)), dict(y=fake(2, 3, 5)), dict(last=fake(2, 4, 4)), dict(x=fake(3, 4))):
        refuse(ValueError, model.causal_conv, **{"x": x, "weight": w, **kw})
    for kw in (dict(weight=fake(4, 4, dtype=torch.float16)), dict(bias=fake(4, dtype=torch.bfloat16)),
               dict(state=fake(2, 3, 4, dtype=torch.float16)), dict(x=fake(2, 3, 4, dtype=torch.int32))):
        refuse(TypeError, model.causal_conv, **{"x": x, "weight": w, **kw})
    refuse(TypeError, model.causal_conv, x, None)
    refuse(ValueError, model.causal_conv_grad, x, w, fake(2, 3, 3))
    refuse(ValueError, model.causal_conv_grad, x, w, x, dlast=fake(2, 2, 4))


def test_clip_lists():
    x = fake(3, 4)
    refuse(ValueError, model.clip_grad_norm, [], 1.0)
    refuse(ValueError, model.clip_grad_norm, [x], 1.0, out=[x, x])
    refuse(ValueError, model.clip_grad_norm, [x], 1.0, out=[fake(4, 3)])
    refuse(ValueError, model.clip_grad_norm, [fake(4, 3).t()], 1.0)
    refuse(TypeError, model.clip_grad_norm, [fake(3, dtype=torch.float64)], 1.0)
    refuse(TypeError, model.clip_grad_norm, [x], 1.0, out=[fake(3, 4, dtype=torch.int32)])
    refuse(TypeError, model.clip_grad_norm, [x, None], 1.0)


def test_beam_shapes_and_types():
    z, s = fake(2, 3, 7), fake(2, 3)
    refuse(ValueError, model.beam_select, fake(2, 7), s)
    refuse(ValueError, model.beam_select, z, fake(2, 4))
    refuse(TypeError, model.beam_select, z, fake(2, 3, dtype=torch.float64))
    refuse(TypeError, model.beam_select, z, s, last=fake(2, 3, dtype=torch.int32))
    refuse(TypeError, model.beam_select, fake(2, 3, 7, dtype=torch.int64), s)
    refuse(ValueError, model.beam_select, fake(2, 7, 3).transpose(1, 2), s)
    p = fake(2, 5, dtype=torch.int32)
    refuse(TypeError, model.beam_reorder, [z], fake(2, 5, dtype=torch.int64))
    refuse(TypeError, model.beam_reorder, [z], None)
    refuse(TypeError, model.beam_reorder, [None], p)
    refuse(ValueError, model.beam_reorder, [z], p[0])
    refuse(ValueError, model.beam_reorder, [z, fake(2, 4, 7)], p)
    refuse(ValueError, model.beam_reorder, [fake(3, 3)], p)
    refuse(ValueError, model.beam_reorder, [z], p, out=[fake(2, 5, 6)])
    refuse(TypeError, model.beam_reorder, [z], p, out=[fake(2, 5, 7, dtype=torch.float16)])
    refuse(ValueError, model.beam_reorder, [z], p, out=[])
    refuse(ValueError, model.beam_reorder, [fake(2, 7, 3).transpose(1, 2)], p)
    assert model.beam_reorder([], p) == []
