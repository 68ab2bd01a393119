"""Calls of the operators of selective models at the ends of what the header
allows, without a GPU."""
import pytest
import torch

from paper_2003_02989_amd import model
from test_model_binding_cpu import fake


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
