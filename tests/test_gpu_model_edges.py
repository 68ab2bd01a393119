"""The operators of selective models at the ends of what the header allows: sizes
of nothing and values near the largest ones."""
import pytest
import torch

from paper_2003_02989_amd import model
from paper_2003_02989_amd.records import SelectiveRecordModel, ising_records
from test_gpu_seq import TYPES, U, check, rounded

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


@pytest.mark.parametrize("n", [4, 5003, 300000])
@pytest.mark.parametrize("max_norm,scale", [(1.0, 1.0), (1e-10, 1e-30), (2.0 ** -120, 2.0 ** -20), (1e-3, 3.0)])
def test_clipping_by_factors_below_the_normal_numbers(n, max_norm, scale):
    """Elements near the largest value and a norm above it: the factor is no normal
    fp32 number, the outputs are; they are as near as with any other factor."""
    kinds = list(TYPES.values())
    sign = torch.where(torch.arange(n) % 3 == 1, -1.0, 1.0)
    values = [(3e38 * sign).to(torch.float32), (1e38 * sign).to(torch.bfloat16), torch.full((5,), 6e4).to(torch.float16)]
    total = sum(float((v.double() ** 2).sum()) for v in values)
    factor = float(torch.tensor(max_norm).double()) / total ** 0.5  # of the elements: the scale is in the norm too
    for swap in range(3):
        outs = [torch.full(v.shape, 9.0, dtype=kinds[(k + swap) % 3][0], device="cuda") for k, v in enumerate(values)]
        norm, _ = model.clip_grad_norm([v.cuda() for v in values], max_norm, scale=scale, out=outs)
        want_norm = torch.tensor(float(torch.tensor(scale).double()) * total ** 0.5, dtype=torch.float64).float()
        assert torch.isclose(norm.cpu(), want_norm, rtol=2 * U, atol=0)
        for k, (o, v) in enumerate(zip(outs, values)):
            w = v.double() * factor
            _, u, tiny = kinds[(k + swap) % 3]
            # the factor, the product and the output's type, each rounded once
            check("output", o, w.numpy(), rounded(w.numpy(), 2.1 * U * w.abs().numpy() + 2.0 ** -149, u, tiny))
    grads = [v.cuda() for v in values]
    model.clip_grad_norm(grads, max_norm, scale=scale)
    for k, (o, v) in enumerate(zip(grads, values)):
        w = v.double() * factor
        _, u, tiny = kinds[k]
        check("in place", o, w.numpy(), rounded(w.numpy(), 2.1 * U * w.abs().numpy() + 2.0 ** -149, u, tiny))


def test_clipping_by_an_infinite_bound():
    """max_norm = infinity cuts nothing, whatever the norm: the elements are scaled."""
    g = torch.tensor([3e38, -3e38, float("inf"), 0.0], device="cuda")
    norm, (o,) = model.clip_grad_norm([g], float("inf"), scale=0.5, out=[torch.empty_like(g)])
    assert float(norm) == float("inf") and torch.equal(o, g * 0.5)
    norm, (o,) = model.clip_grad_norm([g[:2]], float("inf"), out=[torch.empty_like(g[:2])])
    assert float(norm) == float("inf") and torch.equal(o, g[:2])  # 4.2e38 is no fp32 number


@pytest.mark.parametrize("taps", [1, 2])
def test_search_with_few_taps(taps):
    """A convolution of one tap carries no inputs along: its state has no elements.
    With a beam for every continuation the scores are those of all of them."""
    n, R, steps = 1, 2, 3
    m = SelectiveRecordModel(n, 16, states=3, taps=taps, dtype=torch.float32, seed=5)
    m.params["readout"] *= 40
    records = ising_records(n, 6, R, seed=3)
    scores, found = m.most_likely(records, steps, 2 ** steps)
    assert found.shape == (R, 2 ** steps, steps)
    p = m.working()
    for r in range(R):
        rows = torch.cat((records[r].expand(2 ** steps, -1), found[r]), 1)
        y = m.advance(m.inputs(rows), m.beginning(2 ** steps), p)
        z = (y.double() @ p["readout"].double().t())[..., :2]
        want = torch.log_softmax(z, -1).gather(-1, rows[..., None])[:, 6:, 0].sum(1)
        # sums of three scores in fp32, of logits that are fp32 products of 16
        assert torch.allclose(scores[r].double(), want, atol=1e-4, rtol=1e-5)
        assert len({tuple(f) for f in found[r].tolist()}) == 2 ** steps


@pytest.mark.parametrize("taps", [1, 4])
def test_search_of_no_records(taps):
    m = SelectiveRecordModel(2, 16, states=3, taps=taps, dtype=torch.float32, seed=5)
    none = torch.zeros((0, 6), dtype=torch.int64, device="cuda")
    scores, found = m.most_likely(none, 2, 3)
    assert scores.shape == (0, 3) and found.shape == (0, 3, 2)
    scores, found = m.most_likely(none, 0, 3)
    assert found.shape[0] == 0 and found.shape[2] == 0
