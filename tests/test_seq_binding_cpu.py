"""The sequence binding's own argument checks, without a GPU."""
import pytest
import torch

from paper_2003_02989_amd import records, seq


def test_rows_of_strided_tensors():
    class Fake(torch.Tensor):  # stands for a device tensor
        is_cuda = True

    def fake(t):
        return t.as_subclass(Fake)
    x = fake(torch.zeros((4, 6, 10)))
    assert seq._rows(x, "x")[1] == 10
    assert seq._rows(fake(torch.zeros((5, 12))[:, :7]), "x")[1] == 12
    assert seq._rows(fake(torch.zeros((3, 4, 12))[..., 3:9]), "x")[1] == 12
    for bad in (torch.zeros((4, 6)).t(), torch.zeros((4, 6, 10)).transpose(0, 1), torch.zeros((4, 8))[:, ::2],
                torch.zeros((1, 5)).expand(3, 5)):
        with pytest.raises(ValueError):
            seq._rows(fake(bad), "x")
    with pytest.raises(ValueError):
        seq._rows(fake(torch.zeros(())), "x")
    assert seq._steps(fake(torch.zeros((2, 3, 8))[..., :4]), "x", None, (2, 3, 4))[1:] == (24, 8)
    with pytest.raises(ValueError):
        seq._steps(fake(torch.zeros((2, 3, 8))[..., ::2]), "x", None, (2, 3, 4))
    with pytest.raises(ValueError):
        seq._dense(fake(torch.zeros((4, 4)).t()), "x", torch.float32)
    with pytest.raises(TypeError):
        seq._dense(fake(torch.zeros(3)), "x", torch.int64)


def test_records_module_imports():
    assert records.RecordModel and records.ising_records


def test_tensors_of_another_device_are_refused(monkeypatch):
    class On(torch.Tensor):  # stands for a tensor of device `at`
        is_cuda = True
        at = 0

        def get_device(self):
            return self.at

    def on(t, at):
        t = t.as_subclass(On)
        t.at = at
        return t
    monkeypatch.setattr(seq, "_many", True, raising=False)
    monkeypatch.setattr(seq, "_device", lambda: 0, raising=False)
    x = torch.zeros((2, 3, 4))
    for take in (lambda t: seq._dense(t, "x", torch.float32), lambda t: seq._rows(t, "x"),
                 lambda t: seq._steps(t, "x", None, (2, 3, 4))):
        take(on(x, 0))
        with pytest.raises(ValueError, match="device 1"):
            take(on(x, 1))
    assert seq._typed(on(x, 0), "x") == (0, 0)
    with pytest.raises(ValueError, match="device 1"):
        seq._typed(on(x, 1), "x")
