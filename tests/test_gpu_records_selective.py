"""The selective model of measurement records: the operators of selective models
run together, from the sampler's bitstrings through a training step to the most
likely records."""
import itertools
import math

import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import model as ref
from oracle import seq as sref
from paper_2003_02989_amd.records import SelectiveRecordModel, ising_records

pytestmark = pytest.mark.gpu


def oracle_loss(model, records, lengths):
    """Loss and gradients in 64 bits, from the oracle's forms."""
    p = {k: v.double().cpu().numpy() for k, v in model.working().items()}
    rec = records.cpu().numpy()
    B, T = rec.shape
    W, S = model.width, model.states
    ids = np.concatenate([np.full((B, 1), model.start), rec[:, :-1]], 1)
    n = np.full(B, T) if lengths is None else lengths.cpu().numpy()
    e = sref.embed(ids, p["table"], 1.0).reshape(B, T, 3 * W + 2 * S)
    x, dt, z, Bm, Cm = np.split(e, np.cumsum([W, W, W, S]), 2)
    u = ref.causal_conv(x, p["taps"], p["tap_bias"], None, n, True)[0]
    args = (u, dt, p["A"], Bm, Cm, p["skip"], z, p["dt_bias"], None, n)
    h = ref.selective_scan(*args)[0].reshape(B * T, W)
    y = sref.norm(h, p["weight"], p["bias"], 1e-5)[0]
    there = (rec >= 0) & (np.arange(T) < n[:, None])
    up = there.ravel() / max(there.sum(), 1)
    dy, dread, loss, _, _ = sref.xent_grad(y, p["readout"], np.where(there, rec, -1).ravel(), up)
    dh, dw, db = sref.norm_grad(h, p["weight"], 1e-5, dy)
    g = ref.selective_scan_grad(*args, dh.reshape(B, T, W), None)
    dx, dtaps, dtb, _ = ref.causal_conv_grad(x, p["taps"], p["tap_bias"], None, n, True, g[0], None)
    de = np.concatenate([dx, g[1], g[6], g[3], g[4]], 2)
    dtable = sref.embed_grad(ids, de.reshape(B * T, -1), model.vocab, 1.0)[0]
    return (loss * up).sum(), {"table": dtable, "taps": dtaps, "tap_bias": dtb, "log_A": g[2] * p["A"], "skip": g[5],
                               "dt_bias": g[7], "weight": dw, "bias": db, "readout": dread}


# of the numbers between the shots and a gradient, some fourteen tensors are rounded
# to half a unit u of the type, factors of up to four from one to the next; in fp32
# the sums of a few hundred terms count as many again
@pytest.mark.parametrize("dtype,u", [(torch.float32, 2.0 ** -24 * 100), (torch.bfloat16, 2.0 ** -8), (torch.float16, 2.0 ** -11)])
@pytest.mark.parametrize("ragged", [False, True])
def test_loss_and_gradients(dtype, u, ragged):
    records = ising_records(4, 37, 9, seed=3)
    lengths = None
    if ragged:
        lengths = torch.tensor([37, 0, 1, 16, 17, 33, 37, 2, 36], dtype=torch.int32, device="cuda")
        records[3, 5] = -1
    model = SelectiveRecordModel(4, 24, states=5, dtype=dtype, seed=1)
    loss, grads = model.loss_and_grads(records, lengths)
    wl, wg = oracle_loss(model, records, lengths)
    assert abs(float(loss) - wl) <= 56 * u * wl
    for k, g in grads.items():
        assert g.dtype == torch.float32 and g.shape == model.params[k].shape
        g = g.double().cpu().numpy()
        err = np.linalg.norm(g - wg[k]) / np.linalg.norm(wg[k])
        say(str(dtype), k, "error", err)
        assert err <= 56 * u, k


def test_gradients_match_differences_of_the_loss():
    """The loss itself, moved along each parameter's gradient."""
    records = ising_records(3, 40, 16, seed=4)
    model = SelectiveRecordModel(3, 24, states=4, dtype=torch.float32, seed=2)
    _, grads = model.loss_and_grads(records)
    for k, g in grads.items():
        g = g.double()
        eps = 1e-2 / float(g.norm())
        keep = model.params[k].clone()
        value = []
        for s in (1, -1):
            model.params[k] = (keep.double() + s * eps * g).float()
            value.append(float(model.loss_and_grads(records)[0].double()))
        model.params[k] = keep
        # moved by 1e-2 in all: curvature of order one leaves 1e-4 relative, fp32
        # losses of about 2 leave 4e-7 / (2e-2 |g|)
        got, want = (value[0] - value[1]) / (2 * eps), float((g * g).sum())
        say(k, got, want)
        assert abs(got - want) <= 2e-3 * want + 4e-5 * float(g.norm()), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_a_step_cuts_the_gradients(dtype):
    records = ising_records(4, 20, 64, seed=8)
    model = SelectiveRecordModel(4, 32, states=3, dtype=dtype, seed=9)
    _, grads = model.loss_and_grads(records)
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads.values()))
    _, cut = model.loss_and_grads(records, max_norm=norm / 4)
    for k in grads:  # fp32 products of the same gradients with two factors
        assert torch.allclose(cut[k], grads[k] / 4, rtol=1e-6, atol=0), k
    before = {k: p.clone() for k, p in model.params.items()}
    model.step(records)
    for k, p in model.params.items():
        assert torch.isfinite(p).all() and not torch.equal(p, before[k]), k


def test_serving_step_by_step_matches_the_sequence():
    n, B, T = 5, 7, 30
    records = ising_records(n, T, B, seed=6)
    records[2, 4] = -1
    model = SelectiveRecordModel(n, 40, dtype=torch.float32, seed=7)
    p, ids = model.working(), model.inputs(records)
    state = model.beginning(B)
    y = model.advance(ids, state, p)
    z = y.double() @ p["readout"].double().t()
    want = torch.logsumexp(z, -1) - z.gather(-1, records.clamp(min=0)[..., None])[..., 0]
    want[records < 0] = 0
    step = model.beginning(B)
    got = torch.stack([model.score(ids[:, t], records[:, t].contiguous(), step, p) for t in range(T)], 1)
    # fp32 through the chain, states of up to 30 steps in another order: 1e-5 of
    # normalised states of order one, in logits of 40 products of 0.02
    assert torch.allclose(got.double(), want, atol=1e-4)
    for a, b in zip(state, step):
        assert torch.allclose(a.float(), b.float(), rtol=1e-4, atol=1e-5)
    assert got[2, 4] == 0


def test_search_finds_the_most_likely_records():
    """With a beam for every continuation a search is exhaustive: the scores of
    all continuations, formed one by one, in order."""
    n, R, steps = 1, 3, 5
    model = SelectiveRecordModel(n, 16, states=3, dtype=torch.float32, seed=11)
    model.params["readout"] *= 40
    records = ising_records(n, 6, R, seed=12)
    beams = 2 ** steps
    scores, found = model.most_likely(records, steps, beams)
    p = model.working()
    every = list(itertools.product(range(2), repeat=steps))
    for r in range(R):
        rows = torch.cat((records[r].expand(len(every), -1), torch.tensor(every, device="cuda")), 1)
        y = model.advance(model.inputs(rows), model.beginning(len(every)), p)
        z = (y.double() @ p["readout"].double().t())[..., :2]
        logp = torch.log_softmax(z, -1).gather(-1, rows[..., None])[:, 6:, 0].sum(1)
        best, order = logp.sort(descending=True)
        # sums of five scores in fp32, of logits that are fp32 products of 16
        assert torch.allclose(scores[r].double(), best, atol=1e-4, rtol=1e-5)
        for k, f in enumerate(found[r].tolist()):
            assert abs(float(logp[every.index(tuple(f))]) - float(best[k])) <= 2e-4
        assert len({tuple(f) for f in found[r].tolist()}) == beams
    few_scores, few = model.most_likely(records, steps, 4)
    assert few.shape == (R, 4, steps) and torch.all(few_scores <= scores[:, :4] + 1e-4)
    assert model.most_likely(records[:, :0], 2, 3)[1].shape == (R, 3, 2)
