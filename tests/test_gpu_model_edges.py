"""The operators of selective models at the ends of what the header allows: sizes
of nothing and values near the largest ones."""
import pytest
import torch

from paper_2003_02989_amd import model
from test_gpu_seq import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("ragged", [False, True])
def test_scan_gradient_of_no_channels(ty, ragged):
    """dB and dC are sums over no channels: zeros, also where they are views and on
    a stream of the caller's."""
    dtype = TYPES[ty][0]
    new = dict(device="cuda", dtype=dtype)
    x, s, A = torch.zeros((3, 40, 0), **new), torch.ones((3, 40, 5), **new), torch.zeros((0, 5), device="cuda")
    lengths = torch.tensor([0, 40, 7], dtype=torch.int32, device="cuda") if ragged else None
    y, h, states = model.selective_scan(x, x, A, s, s, keep=True, lengths=lengths)
    assert y.shape == (3, 40, 0) and h.shape == (3, 0, 5) and states.shape == (3, 3, 5, 0)
    room = torch.full((3, 40, 12), float("nan"), **new)
    g = model.selective_scan_grad(x, x, A, s, s, states, x, lengths=lengths, dB=room[..., :5], dC=room[..., 5:10])
    assert torch.all(room[..., :10] == 0) and torch.isnan(room[..., 10:]).all()
    assert g.dA.shape == (0, 5) and g.dx.shape == (3, 40, 0) and g.dh0.shape == (3, 0, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = model.selective_scan_grad(x, x, A, s, s, states, x, lengths=lengths, stream=side)
    side.synchronize()
    assert torch.all(g.dB == 0) and torch.all(g.dC == 0)
