"""The recurrent model of measurement records: the sequence operators chained
from the sampler's bitstrings to the loss and back."""
import math

import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import oracle as orc
from oracle import seq as ref
from paper_2003_02989_amd import seq
from paper_2003_02989_amd.records import RecordModel, ising_records

pytestmark = pytest.mark.gpu


def oracle_loss(model, records, lengths):
    """Loss and gradients of the model in 64 bits, from the oracle's forms."""
    p = {k: v.double().cpu().numpy() for k, v in model.working().items()}
    rec = records.cpu().numpy()
    B, T = rec.shape
    W = model.width
    ids = np.concatenate([np.full((B, 1), model.start), rec[:, :-1]], 1)
    n = np.full(B, T) if lengths is None else lengths.cpu().numpy()
    e = ref.embed(ids, p["table"], 1.0).reshape(B, T, 2 * W)
    h = ref.scan(e[..., :W], e[..., W:], None, n)[0]
    flat = h.reshape(B * T, W)
    y = ref.norm(flat, p["weight"], p["bias"], 1e-5)[0]
    there = (rec >= 0) & (np.arange(T) < n[:, None])
    up = there.ravel() / max(there.sum(), 1)
    dy, dread, loss, _, _ = ref.xent_grad(y, p["readout"], np.where(there, rec, -1).ravel(), up)
    dh, dw, db = ref.norm_grad(flat, p["weight"], 1e-5, dy)
    dx, dg = ref.scan_grad(e[..., :W], e[..., W:], None, n, dh.reshape(B, T, W), None)[:2]
    dt = ref.embed_grad(ids, np.concatenate([dx, dg], 2).reshape(B * T, 2 * W), model.vocab, 1.0)[0]
    return (loss * up).sum(), {"table": dt, "weight": dw, "bias": db, "readout": dread}


@pytest.mark.parametrize("ragged", [False, True])
def test_loss_and_gradients_in_fp32(ragged):
    records = ising_records(4, 70, 9, seed=3)
    lengths = None
    if ragged:
        lengths = torch.tensor([70, 0, 1, 64, 65, 33, 70, 2, 69], dtype=torch.int32, device="cuda")
        records[3, 5] = -1
    model = RecordModel(4, 40, dtype=torch.float32, seed=1)
    loss, grads = model.loss_and_grads(records, lengths)
    wl, wg = oracle_loss(model, records, lengths)
    # fp32 rounding through the chain: sums of up to 630 terms of order one and
    # a few hundred operations each way, 2^-24 each, against gradients whose
    # largest entry sets the scale
    assert abs(float(loss) - wl) <= 2e-5 * abs(wl)
    for k in grads:
        g = grads[k].double().cpu().numpy()
        err = np.abs(g - wg[k]).max() / np.abs(wg[k]).max()
        say(k, "error", err)
        assert err <= 2e-4, k


def test_gradients_match_differences_of_the_loss():
    """The loss itself, moved along each parameter's gradient."""
    records = ising_records(3, 40, 16, seed=4)
    model = RecordModel(3, 24, dtype=torch.float32, seed=2)
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


def test_training_learns_the_records_distribution():
    """The loss falls below that of uniform bitstrings, to near the entropy of
    the circuits' own distributions."""
    n, steps = 4, 16
    model = RecordModel(n, 64, seed=5)
    first = last = None
    for i in range(120):
        loss = model.step(ising_records(n, steps, 512, seed=i), lr=2e-2)
        first = float(loss) if i == 0 else first
    last = float(loss)
    # entropy of the measured distributions, from the shots of many records
    shots = ising_records(n, steps, 20000, seed=999).cpu().numpy()
    entropy = 0.0
    for t in range(steps):
        p = np.bincount(shots[:, t], minlength=1 << n) / shots.shape[0]
        entropy -= (p[p > 0] * np.log(p[p > 0])).sum() / steps
    say("first", first, "last", last, "entropy", entropy, "uniform", math.log(1 << n))
    assert first > last and last < 0.5 * (math.log(1 << n) + entropy)


def test_serving_step_by_step_matches_the_sequence():
    n, B, T = 5, 7, 30
    records = ising_records(n, T, B, seed=6)
    records[2, 4] = -1
    model = RecordModel(n, 80, seed=7)
    p, ids = model.working(), model.inputs(records)
    W = model.width
    e = seq.embed(ids, p["table"])
    h, h_last = seq.gated_scan(e[..., :W], e[..., W:])
    loss = seq.softmax_xent(seq.layer_norm(h, p["weight"], p["bias"]), p["readout"], records)[0]
    state = torch.zeros((B, W), device="cuda")
    steps = torch.stack([model.score(ids[:, t], records[:, t].contiguous(), state, p) for t in range(T)], 1)
    # the same formulas in another order: bf16 states may round the other way,
    # 2^-8 of states of at most 4 in logits summed over 80 products of 0.02
    assert torch.allclose(steps, loss, atol=2e-2)
    assert torch.allclose(state, h_last, rtol=1e-5, atol=1e-5)
    assert steps[2, 4] == 0
