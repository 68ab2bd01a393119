"""Models of measurement records, trained on what circuits answer.

    python -m paper_2003_02989_amd.records [--model recurrent|selective] [--qubits 8] [--records 512] [--steps 48]
                                           [--iters 200]

A record is one measured bitstring per time step of a quantum system's
evolution; here a transverse-field Ising chain in first-order Trotter steps, as
a batch of circuits with the time in their symbols (``ising_records``).
``RecordModel`` learns the distribution of the next bitstring from those before
it, as the paper's hybrid examples put a classical recurrent network beside
the circuits:

    table lookup of the bitstring -> x, g        (seq.embed)
    h_t = a_t h_{t-1} + (1 - a_t) x_t, a = sigmoid(g)   (seq.gated_scan)
    layer norm of the states                      (seq.layer_norm)
    cross entropy over all bitstrings             (seq.softmax_xent)

``SelectiveRecordModel`` has a state space in place of the recurrence:

    table lookup of the bitstring -> x, dt, z, B, C          (seq.embed)
    x mixed with the steps before it                         (model.causal_conv)
    h_t = exp(d_t A) h_{t-1} + d_t x_t B_t, y_t = C_t . h_t  (model.selective_scan)
    layer norm and cross entropy as above

is trained with clipped gradients (model.clip_grad_norm) and answers with the most
likely records (model.beam_select, model.beam_reorder).

The bitstrings go from the sampler to the table as they are; the id 2^n is the
start of a record, and -1, the marker of a missing shot, has no embedding and no
loss.
"""
import argparse
import math

import torch

from . import model as ops
from . import seq, tq
from .circuits import Circuit, program_blob, sym


def ising_records(n, steps, records, seed, dt=0.25, field=0.9):
    """int64 [records, steps]: one shot of a chain of n qubits at each of the
    times dt, 2 dt, ... steps dt, evolved from |0...0>.  Row t of the batch is
    the circuit of time (t + 1) dt in n Trotter steps; all records' shots at that
    time come from one simulation."""
    c = Circuit(n)
    for _ in range(n):
        for q in range(n - 1):
            c.add("RZZ", (q, q + 1), [sym(0, -2.0 / n)])
        for q in range(n):
            c.add("RX", q, [sym(0, -2.0 * field / n)])
    prog = tq.Program(program_blob([c] * steps, 1), specialize=True)
    time = dt * torch.arange(1, steps + 1, dtype=torch.float32, device="cuda")[:, None]
    shots = tq.sample(prog, time, records, seed)
    return shots.t().contiguous()


class RecordModel:
    """Parameters and one training step; ``dtype`` is that of the parameters'
    working copies and of the activations, the parameters themselves are fp32.

    float16 has no numbers below 2^-24, where the terms of a mean over many shots
    lie: its loss is scaled before the gradients are formed, and they are given
    back in fp32, without the scale."""

    def __init__(self, n, width, dtype=torch.bfloat16, seed=0):
        self.start, self.width, self.dtype = 1 << n, width, dtype
        self.vocab = self.start + 1
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(shape, device="cuda", generator=gen) * std
        self.params = {
            "table": normal(self.vocab, 2 * width, std=1.0),
            "weight": torch.ones(width, device="cuda"),
            "bias": torch.zeros(width, device="cuda"),
            "readout": normal(self.vocab, width, std=0.02),
        }
        self.params["table"][:, width:] += 2.0  # gates begin near one: memories of several steps
        self.moments = {k: (torch.zeros_like(p), torch.zeros_like(p)) for k, p in self.params.items()}
        self.t = 0

    def working(self):
        return {k: p.to(self.dtype) for k, p in self.params.items()}

    def inputs(self, records):
        """The id before each one of the records: the start, then the records."""
        first = torch.full_like(records[:, :1], self.start)
        return torch.cat((first, records[:, :-1]), 1)

    def loss_scale(self, shots):
        """A power of two near the root of the number of shots: a shot's part of the
        gradients is that much above their mean, their sum that much below what it
        would be without a mean."""
        return 2.0 ** (shots.bit_length() // 2) if self.dtype == torch.float16 else 1.0

    def loss_and_grads(self, records, lengths=None):
        """(mean loss of the shots there are, gradients in ``dtype``, of float16 in
        fp32); records [B, T], -1 where there is no shot, lengths int32 [B] or
        None."""
        p, W = self.working(), self.width
        ids = self.inputs(records)
        e = seq.embed(ids, p["table"])
        h, _, kept = seq.gated_scan(e[..., :W], e[..., W:], lengths=lengths, keep=True)
        y, mean, rstd = seq.layer_norm(h, p["weight"], p["bias"], keep=True)
        there = records >= 0
        if lengths is not None:
            there &= torch.arange(records.shape[1], device=records.device) < lengths[:, None]
        targets = torch.where(there, records, torch.full_like(records, -1))
        count = there.sum().clamp(min=1).float()
        scale = self.loss_scale(records.numel())
        upstream = there.float() / count * scale
        dy, dreadout, loss, _ = seq.softmax_xent_grad(y, p["readout"], targets, upstream)
        dh, dweight, dbias = seq.layer_norm_grad(h, p["weight"], mean, rstd, dy)
        de = torch.empty_like(e)
        seq.gated_scan_grad(e[..., :W], e[..., W:], kept, dh, lengths=lengths, dx=de[..., :W], dg=de[..., W:])
        dtable = seq.embed_grad(ids, de, self.vocab)
        grads = {"table": dtable, "weight": dweight, "bias": dbias, "readout": dreadout}
        if self.dtype == torch.float16:
            grads = {k: g.float() / scale for k, g in grads.items()}
        return loss.sum() / count, grads

    def step(self, records, lengths=None, lr=1e-2):
        """One Adam step; returns the loss before it (a device scalar)."""
        loss, grads = self.loss_and_grads(records, lengths)
        self.update(grads, lr)
        return loss

    def update(self, grads, lr):
        self.t += 1
        for k, g in grads.items():
            g = g.float()
            m, v = self.moments[k]
            m.lerp_(g, 0.1)
            v.lerp_(g * g, 0.01)
            rate = lr * (1 - 0.99 ** self.t) ** 0.5 / (1 - 0.9 ** self.t)
            self.params[k].addcdiv_(m, v.sqrt().add_(1e-8), value=-rate)

    def score(self, ids, targets, h, p=None):
        """One step of serving: takes the ids [B] that the records have reached,
        advances their states h [B, width] in place and returns the negative log
        likelihood [B] of ``targets`` as the next ones."""
        p = p or self.working()
        e, W = seq.embed(ids[:, None].contiguous(), p["table"]), self.width
        y, _ = seq.gated_scan(e[..., :W], e[..., W:], h, h_last=h)
        y = seq.layer_norm(y, p["weight"], p["bias"])
        return seq.softmax_xent(y[:, 0], p["readout"], targets.contiguous())[0]


class SelectiveRecordModel(RecordModel):
    """Parameters and one training step of the selective model with ``states``
    states per channel and a convolution of ``taps`` steps; A = -exp(log_A) and what
    else the scan holds in fp32 have no working copies."""

    def __init__(self, n, width, states=16, taps=4, dtype=torch.bfloat16, seed=0):
        self.start, self.width, self.states, self.taps, self.dtype = 1 << n, width, states, taps, dtype
        self.vocab = self.start + 1
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(shape, device="cuda", generator=gen) * std
        # steps of 0.001 to 0.1 to begin with, decays of 1 to `states`
        step = torch.exp(torch.rand(width, device="cuda", generator=gen) * math.log(100.0) + math.log(1e-3))
        decay = torch.arange(1, states + 1, device="cuda", dtype=torch.float32)
        self.params = {
            "table": normal(self.vocab, 3 * width + 2 * states, std=1.0),
            "taps": normal(taps, width, std=1 / math.sqrt(taps)),
            "tap_bias": torch.zeros(width, device="cuda"),
            "log_A": decay.log().expand(width, states).contiguous(),
            "skip": torch.ones(width, device="cuda"),
            "dt_bias": torch.log(torch.expm1(step)),
            "weight": torch.ones(width, device="cuda"),
            "bias": torch.zeros(width, device="cuda"),
            "readout": normal(self.vocab, width, std=0.02),
        }
        self.moments = {k: (torch.zeros_like(p), torch.zeros_like(p)) for k, p in self.params.items()}
        self.t = 0

    def working(self):
        held = ("log_A", "skip", "dt_bias")
        p = {k: v if k in held else v.to(self.dtype) for k, v in self.params.items()}
        p["A"] = -torch.exp(p["log_A"])
        return p

    def parts(self, e):
        """x, dt, z, B, C of looked-up rows."""
        W, S = self.width, self.states
        return e.split((W, W, W, S, S), -1)

    def loss_and_grads(self, records, lengths=None, max_norm=math.inf):
        """(mean loss of the shots there are, gradients in fp32 cut to max_norm);
        records [B, T], -1 where there is no shot, lengths int32 [B] or None."""
        p = self.working()
        ids = self.inputs(records)
        e = seq.embed(ids, p["table"])
        x, dt, z, B, C = self.parts(e)
        u, _ = ops.causal_conv(x, p["taps"], bias=p["tap_bias"], lengths=lengths)
        scan = (u, dt, p["A"], B, C)
        more = dict(skip=p["skip"], z=z, dt_bias=p["dt_bias"], lengths=lengths)
        h, _, kept = ops.selective_scan(*scan, keep=True, **more)
        y, mean, rstd = seq.layer_norm(h, p["weight"], p["bias"], keep=True)
        there = records >= 0
        if lengths is not None:
            there &= torch.arange(records.shape[1], device=records.device) < lengths[:, None]
        targets = torch.where(there, records, torch.full_like(records, -1))
        count = there.sum().clamp(min=1).float()
        scale = self.loss_scale(records.numel())
        dy, dreadout, loss, _ = seq.softmax_xent_grad(y, p["readout"], targets, there.float() / count * scale)
        dh, dweight, dbias = seq.layer_norm_grad(h, p["weight"], mean, rstd, dy)
        de = torch.empty_like(e)
        dx, ddt, dz, dB, dC = self.parts(de)
        g = ops.selective_scan_grad(*scan, kept, dh, ddt=ddt, dz=dz, dB=dB, dC=dC, **more)
        c = ops.causal_conv_grad(x, p["taps"], g.dx, bias=p["tap_bias"], lengths=lengths, dx=dx)
        grads = {"table": seq.embed_grad(ids, de, self.vocab), "taps": c.dweight, "tap_bias": c.dbias,
                 "log_A": g.dA * p["A"], "skip": g.dskip, "dt_bias": g.ddt_bias, "weight": dweight, "bias": dbias,
                 "readout": dreadout}
        outs = [torch.empty_like(self.params[k]) for k in grads]
        ops.clip_grad_norm(list(grads.values()), max_norm, scale=1 / scale, out=outs)
        return loss.sum() / count, dict(zip(grads, outs))

    def step(self, records, lengths=None, lr=1e-2, max_norm=1.0):
        """One Adam step with gradients cut to max_norm; returns the loss before it
        (a device scalar)."""
        loss, grads = self.loss_and_grads(records, lengths, max_norm)
        self.update(grads, lr)
        return loss

    def beginning(self, records):
        """The states [records, ...] of records that have not begun: what the
        convolution and the scan carry."""
        return [torch.zeros((records, self.taps - 1, self.width), dtype=self.dtype, device="cuda"),
                torch.zeros((records, self.width, self.states), device="cuda")]

    def advance(self, ids, state, p):
        """The normalised states [B, T, width] after each of the ids [B, T] that the
        records have reached, whose states it advances in place."""
        x, dt, z, B, C = self.parts(seq.embed(ids, p["table"]))
        u, _ = ops.causal_conv(x, p["taps"], bias=p["tap_bias"], state=state[0], last=state[0])
        h, _ = ops.selective_scan(u, dt, p["A"], B, C, skip=p["skip"], z=z, dt_bias=p["dt_bias"], h0=state[1],
                                  h_last=state[1])
        return seq.layer_norm(h, p["weight"], p["bias"])

    def score(self, ids, targets, h, p=None):
        """One step of serving: takes the ids [B] that the records have reached,
        advances their states h in place and returns the negative log likelihood
        [B] of ``targets`` as the next ones."""
        p = p or self.working()
        y = self.advance(ids[:, None].contiguous(), h, p)
        return seq.softmax_xent(y[:, 0], p["readout"], targets.contiguous())[0]

    def most_likely(self, records, steps, beams):
        """The most likely continuations that a search with ``beams`` beams finds of
        records [R, T] (T may be 0) by ``steps`` bitstrings: (scores [R, beams],
        bitstrings [R, beams, steps]), best first."""
        p = self.working()
        R = records.shape[0]
        readout = p["readout"].float().t()
        state = self.beginning(R)
        first = torch.full((R, 1), self.start, dtype=torch.int64, device=records.device)
        y = self.advance(torch.cat((first, records), 1), state, p)[:, -1:]
        scores = torch.zeros((R, 1), device=records.device)
        found = torch.empty((R, 1, steps), dtype=torch.int64, device=records.device)
        for t in range(steps):
            W = scores.shape[1]
            logits = (y.reshape(-1, self.width).float() @ readout).view(R, W, self.vocab)
            logits[..., self.start] = -math.inf  # not a bitstring
            wide = min(beams, W * self.start)
            scores, parents, tokens = ops.beam_select(logits, scores, beams=wide)
            *state, found = ops.beam_reorder([s.view((R, W) + s.shape[1:]) for s in state] + [found], parents)
            found[..., t] = tokens
            state = [s.flatten(0, 1) for s in state]
            y = self.advance(tokens.view(-1, 1), state, p)
        return scores, found


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--model", choices=("recurrent", "selective"), default="recurrent")
    ap.add_argument("--qubits", type=int, default=8)
    ap.add_argument("--records", type=int, default=512)
    ap.add_argument("--steps", type=int, default=48)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--iters", type=int, default=200)
    a = ap.parse_args()
    selective = a.model == "selective"
    model = (SelectiveRecordModel if selective else RecordModel)(a.qubits, a.width)
    for i in range(a.iters):
        records = ising_records(a.qubits, a.steps, a.records, seed=i)
        loss = model.step(records)
        if i % 20 == 0 or i == a.iters - 1:
            print(f"iteration {i}: {float(loss):.4f} nats per bitstring", flush=True)
    held_out = ising_records(a.qubits, a.steps, a.records, seed=1 << 40)
    p, ids = model.working(), model.inputs(held_out)
    h = model.beginning(a.records) if selective else torch.zeros((a.records, a.width), device="cuda")
    nll = torch.stack([model.score(ids[:, t], held_out[:, t], h, p) for t in range(a.steps)], 1)
    print(f"held out, step by step: {float(nll.mean()):.4f} nats per bitstring", flush=True)
    if selective:
        scores, found = model.most_likely(held_out[:1, :a.steps // 2], min(4, a.steps), 8)
        print(f"after {a.steps // 2} bitstrings of the first record, most likely:", flush=True)
        for s, f in zip(scores[0].tolist()[:3], found[0].tolist()):
            print("  " + " ".join(f"{v:0{a.qubits}b}" for v in f) + f": {s:.4f}", flush=True)


if __name__ == "__main__":
    main()
