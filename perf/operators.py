"""The operators of sequence models over measurement records, as cases to measure.

A record is a sequence of measured bitstrings, the integer ids that the
sampler returns: the vocabulary of an n-qubit circuit is its 2^n bitstrings
and one start token, and the marker 2^64 - 1 (-1 as int64) stands where there
is no shot.  A recurrent model of such records looks the ids up in a table,
runs a gated linear recurrence over time, normalises its states and is trained
by the cross entropy of the next bitstring.  Every case is one of these
operators, forward or with its gradient:

  embed, embed_grad   table lookup with scaling; gradient of the table
  scan, scan_train    h_t = a_t h_{t-1} + (1 - a_t) x_t, a_t = sigmoid(g_t)
  norm, norm_train    layer norm of each row
  xent, xent_grad     softmax cross entropy of hidden @ weight^T

Where ``own`` is false ``run`` computes them in their plain form, in 32 bits
with elementary torch operations; where it is true it calls the framework.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
NO_SHOT = -1


def listed():
    return [
        # looking up one batch of the 4-qubit ansatz' measurements, one shot each, to advance its records: all latency
        {"name": "embed_n4_b16_f32", "op": "embed", "type": "f32", "tokens": 16, "vocab": 17, "dim": 64,
         "shots": "random circuit"},
        # the records of 4096 16-qubit circuits, 64 steps each: the gradient of a table of all bitstrings
        {"name": "embed_grad_n16_262144_bf16", "op": "embed_grad", "type": "bf16", "tokens": 262144, "vocab": 65537,
         "dim": 512, "shots": "random circuit"},
        # shots of circuits near a GHZ state: almost all tokens are two bitstrings; an odd count and width
        {"name": "embed_grad_n10_peaked_f32", "op": "embed_grad", "type": "f32", "tokens": 100003, "vocab": 1025,
         "dim": 200, "shots": "two peaks"},
        # one step of the recurrence for 1024 records that are being extended: a call for a single token
        {"name": "scan_step_b1024_bf16", "op": "scan", "type": "bf16", "batch": 1024, "steps": 1, "dim": 512,
         "ragged": False},
        # one long record (repeated measurement of one device): little to do side by side, a long axis; an odd width
        {"name": "scan_b1_t100001_f32", "op": "scan", "type": "f32", "batch": 1, "steps": 100001, "dim": 331,
         "ragged": False},
        # a training step over records of different lengths, empty ones among them
        {"name": "scan_train_b24_t4099_bf16", "op": "scan_train", "type": "bf16", "batch": 24, "steps": 4099,
         "dim": 1024, "ragged": True},
        # normalising the 200 expectation values of a small batch of circuits
        {"name": "norm_b64_d200_f32", "op": "norm", "type": "f32", "rows": 64, "dim": 200},
        # a training step's normalisation
        {"name": "norm_train_65536_bf16", "op": "norm_train", "type": "bf16", "rows": 65536, "dim": 1024},
        # the same for an odd number of rows and an odd width
        {"name": "norm_train_20011_d331_f16", "op": "norm_train", "type": "f16", "rows": 20011, "dim": 331},
        # how likely the next measured bitstring of four records is: single tokens against the whole vocabulary
        {"name": "xent_n16_4_bf16", "op": "xent", "type": "bf16", "tokens": 4, "vocab": 65537, "dim": 512},
        # a training step over the vocabulary of 12 qubits in 32 bits, an odd number of tokens
        {"name": "xent_grad_n12_4099_f32", "op": "xent_grad", "type": "f32", "tokens": 4099, "vocab": 4097,
         "dim": 512},
        # the largest: a training step over all bitstrings of 16 qubits
        {"name": "xent_grad_n16_8192_bf16", "op": "xent_grad", "type": "bf16", "tokens": 8192, "vocab": 65537,
         "dim": 1024},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A further case: operator, direction, type and sizes over the ranges
    that the listed cases stand for, at most the largest listed one's work."""
    most = {"flops": max(work(c)["flops"] for c in listed()), "bytes": 4 << 30}
    while True:
        op = rng.choice(("embed", "embed_grad", "scan", "scan_train", "norm", "norm_train", "xent", "xent_grad"))
        c = {"op": op, "type": rng.choice(("f32", "bf16", "f16"))}
        if op in ("embed", "embed_grad"):
            c.update(tokens=_log(rng, 1, 1 << 20), vocab=(1 << rng.randint(1, 18)) + 1, dim=_log(rng, 16, 2048),
                     shots=rng.choice(("random circuit", "two peaks", "uniform")))
        elif op in ("scan", "scan_train"):
            c.update(batch=_log(rng, 1, 4096), steps=rng.choice((1, _log(rng, 2, 131072), _log(rng, 2, 131072))),
                     dim=_log(rng, 16, 2048), ragged=rng.random() < 0.5)
        elif op in ("norm", "norm_train"):
            c.update(rows=_log(rng, 1, 1 << 18), dim=_log(rng, 16, 8192))
        else:
            c.update(tokens=_log(rng, 1, 16384), vocab=(1 << rng.randint(4, 17)) + 1, dim=_log(rng, 32, 2048))
        w = work(c)
        # the plain scan keeps some ten arrays in 32 bits: 2^28 elements are 11 GB
        elements = c.get("batch", 0) * c.get("steps", 0) * c["dim"]
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and elements <= 1 << 28:
            return c


def _size(case):
    return 4 if case["type"] == "f32" else 2


def work(case):
    """Each input read once and each output written once; products and sums
    of the formulas."""
    s, op, D = _size(case), case["op"], case["dim"]
    if op in ("embed", "embed_grad"):
        N, V = case["tokens"], case["vocab"]
        rows = min(N, V) if op == "embed" else V
        return {"bytes": 8 * N + (N + rows) * D * s, "flops": N * D}
    if op in ("scan", "scan_train"):
        n = case["batch"] * case["steps"] * D
        state = 4 * case["batch"] * D
        # records of different lengths fill about half of the steps; outputs are written whole
        fill = 0.5 if case["ragged"] else 1.0
        if op == "scan":
            return {"bytes": int(n * s * (2 * fill + 1)) + 2 * state, "flops": int(8 * n * fill)}
        return {"bytes": int(n * s * (3 * fill + 3)) + 4 * state, "flops": int(24 * n * fill)}
    if op in ("norm", "norm_train"):
        n = case["rows"] * D
        if op == "norm":
            return {"bytes": 2 * n * s + 2 * D * s, "flops": 8 * n}
        return {"bytes": 4 * n * s + 4 * D * s, "flops": 22 * n}
    N, V = case["tokens"], case["vocab"]
    if op == "xent":
        return {"bytes": (N + V) * D * s + 16 * N, "flops": 2 * N * V * D}
    return {"bytes": 2 * (N + V) * D * s + 20 * N, "flops": 6 * N * V * D}


# ------------------------------------------------------------------- inputs

def _shots(gen, N, V, kind):
    """Measured bitstrings: ids 0 .. V-2; now and then the start token V-1
    and the marker of a missing shot."""
    dev = gen.device
    if kind == "random circuit":  # probabilities of a random circuit: exponentially distributed
        p = -torch.log1p(-torch.rand(V - 1, device=dev, generator=gen))
        t = torch.multinomial(p + 1e-12, N, replacement=True, generator=gen)
    elif kind == "two peaks":  # a GHZ state with some noise
        t = torch.randint(0, V - 1, (N,), device=dev, generator=gen)
        peak = torch.randint(0, 2, (N,), device=dev, generator=gen) * (V - 2)
        t = torch.where(torch.rand(N, device=dev, generator=gen) < 0.05, t, peak)
    else:
        t = torch.randint(0, V - 1, (N,), device=dev, generator=gen)
    u = torch.rand(N, device=dev, generator=gen)
    t = torch.where(u < 1 / 64, torch.full_like(t, V - 1), t)
    return torch.where(u > 0.99, torch.full_like(t, NO_SHOT), t)


def _normal(gen, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, device=gen.device, generator=gen) * scale + shift).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dt, D = case["op"], TYPES[case["type"]], case["dim"]
    st = {"case": case}
    if op in ("embed", "embed_grad"):
        N, V = case["tokens"], case["vocab"]
        st["tokens"] = _shots(gen, N, V, case["shots"])
        st["scale"] = math.sqrt(D)
        if op == "embed":
            st["table"] = _normal(gen, (V, D), dt, 1 / math.sqrt(D))
        else:
            st["grad_out"] = _normal(gen, (N, D), dt, 0.02)
    elif op in ("scan", "scan_train"):
        B, T = case["batch"], case["steps"]
        # both are halves of the looked-up rows, as the model has them
        both = _normal(gen, (B, T, 2 * D), dt)
        st["x"], st["g"] = both[..., :D], both[..., D:]
        st["g"].mul_(1.5).add_(3.0)  # memories of a few steps to hundreds of them
        st["h0"] = _normal(gen, (B, D), torch.float32)
        st["lengths"] = None
        if case["ragged"]:
            st["lengths"] = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
            st["lengths"][0] = 0
        if op == "scan_train":
            st["dy"] = _normal(gen, (B, T, D), dt)
            st["dh_last"] = _normal(gen, (B, D), torch.float32)
    elif op in ("norm", "norm_train"):
        N = case["rows"]
        st["x"] = _normal(gen, (N, D), dt, 1.5, 0.3)
        st["weight"] = _normal(gen, (D,), dt, 0.1, 1.0)
        st["bias"] = _normal(gen, (D,), dt, 0.1)
        if op == "norm_train":
            st["dy"] = _normal(gen, (N, D), dt)
    else:
        N, V = case["tokens"], case["vocab"]
        st["hidden"] = _normal(gen, (N, D), dt)
        st["weight"] = _normal(gen, (V, D), dt, 1.5 / math.sqrt(D))
        st["targets"] = _shots(gen, N, V, "random circuit")
        if op == "xent_grad":
            valid = st["targets"] != NO_SHOT
            # the mean over the shots there are, in 16 bits with a loss scale
            loss_scale = 1.0 if case["type"] == "f32" else 1024.0
            st["upstream"] = valid.float() * (loss_scale / valid.sum().clamp(min=1).float())
    return st


# -------------------------------------------------------------- plain forms

def _plain_embed(tokens, table, scale):
    ok = (tokens >= 0) & (tokens < table.shape[0])
    rows = table[torch.where(ok, tokens, torch.zeros_like(tokens))].float() * scale
    return torch.where(ok[:, None], rows, torch.zeros_like(rows)).to(table.dtype)


def _plain_embed_grad(tokens, grad_out, V, scale):
    ok = (tokens >= 0) & (tokens < V)
    rows = torch.where(ok[:, None], grad_out.float() * scale, torch.zeros((), device=grad_out.device))
    grad = torch.zeros((V, grad_out.shape[1]), device=grad_out.device)
    grad.index_add_(0, torch.where(ok, tokens, torch.zeros_like(tokens)), rows)
    return grad.to(grad_out.dtype)


def _doubling(a, b):
    """h_t = a_t h_{t-1} + b_t along dim 1 from h = 0, by doubling the span
    each step covers."""
    T, d = a.shape[1], 1
    while d < T:
        b = torch.cat((b[:, :d], a[:, d:] * b[:, :-d] + b[:, d:]), 1)
        a = torch.cat((a[:, :d], a[:, d:] * a[:, :-d]), 1)
        d *= 2
    return b


def _plain_scan(st):
    """(y, h_last, states before each step, gates, the steps there are)"""
    x, g, h0, lengths = st["x"].float(), st["g"].float(), st["h0"], st["lengths"]
    T = x.shape[1]
    on = None
    a, c = torch.sigmoid(g), torch.sigmoid(-g)
    b = c * x
    if lengths is not None:  # steps past the end carry the state on
        on = (torch.arange(T, device=x.device)[None, :] < lengths[:, None])[..., None]
        a = torch.where(on, a, torch.ones((), device=x.device))
        b = torch.where(on, b, torch.zeros((), device=x.device))
    first = (a[:, 0] * h0 + b[:, 0])[:, None]
    h = _doubling(a, torch.cat((first, b[:, 1:]), 1))
    y = h if on is None else torch.where(on, h, torch.zeros((), device=x.device))
    before = torch.cat((h0[:, None], h[:, :-1]), 1)
    return y.to(st["x"].dtype), h[:, -1].clone(), before, a, c, on


def _plain_scan_train(st):
    y, h_last, before, a, c, on = _plain_scan(st)
    dy, zero = st["dy"].float(), torch.zeros((), device=a.device)
    if on is not None:
        dy = torch.where(on, dy, zero)
    # l_t = dy_t + a_{t+1} l_{t+1}, from the last step back
    dy = torch.cat((dy[:, :-1], (dy[:, -1] + st["dh_last"])[:, None]), 1)
    nxt = torch.cat((a[:, 1:], torch.ones_like(a[:, :1])), 1)
    l = _doubling(nxt.flip(1), dy.flip(1)).flip(1)
    dh0 = a[:, 0] * l[:, 0]
    dx, dg = c * l, a * c * (before - st["x"].float()) * l
    if on is not None:
        dx, dg = torch.where(on, dx, zero), torch.where(on, dg, zero)
    dt = st["x"].dtype
    return y, h_last, dx.to(dt), dg.to(dt), dh0


def _plain_norm(st):
    x = st["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    xh = (x - mean) * rstd
    return (xh * st["weight"].float() + st["bias"].float()).to(st["x"].dtype), xh, rstd


def _plain_norm_train(st):
    y, xh, rstd = _plain_norm(st)
    dy, dt = st["dy"].float(), st["x"].dtype
    u = dy * st["weight"].float()
    dx = rstd * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
    return y, dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)


def _plain_xent(st, grad):
    h, W, t = st["hidden"].float(), st["weight"].float(), st["targets"]
    ok = (t >= 0) & (t < W.shape[0])
    at = torch.where(ok, t, torch.zeros_like(t))[:, None]
    logits = h @ W.t()
    top = logits.max(1, keepdim=True).values
    lse = (logits - top).exp().sum(1, keepdim=True).log() + top
    loss = torch.where(ok, (lse - logits.gather(1, at))[:, 0], torch.zeros((), device=h.device))
    if not grad:
        return loss, lse[:, 0]
    up = torch.where(ok, st["upstream"], torch.zeros((), device=h.device))[:, None]
    p = (logits - lse).exp_()
    p.scatter_add_(1, at, torch.full_like(at, -1, dtype=p.dtype))
    p *= up
    dt = st["hidden"].dtype
    return (p @ W).to(dt), (p.t() @ h).to(dt), loss, lse[:, 0]


def run(st):
    if own:
        return _run_own(st)
    op = st["case"]["op"]
    if op == "embed":
        return _plain_embed(st["tokens"], st["table"], st["scale"])
    if op == "embed_grad":
        return _plain_embed_grad(st["tokens"], st["grad_out"], st["case"]["vocab"], st["scale"])
    if op == "scan":
        return _plain_scan(st)[:2]
    if op == "scan_train":
        return _plain_scan_train(st)
    if op == "norm":
        return _plain_norm(st)[0]
    if op == "norm_train":
        return _plain_norm_train(st)
    return _plain_xent(st, op == "xent_grad")


def _run_own(st):
    from paper_2003_02989_amd import seq
    op = st["case"]["op"]
    if op == "embed":
        return seq.embed(st["tokens"], st["table"], scale=st["scale"])
    if op == "embed_grad":
        return seq.embed_grad(st["tokens"], st["grad_out"], st["case"]["vocab"], scale=st["scale"])
    if op == "scan":
        return seq.gated_scan(st["x"], st["g"], st["h0"], lengths=st["lengths"])
    if op == "scan_train":
        y, h_last, states = seq.gated_scan(st["x"], st["g"], st["h0"], lengths=st["lengths"], keep=True)
        dx, dg, dh0 = seq.gated_scan_grad(st["x"], st["g"], states, st["dy"], dh_last=st["dh_last"],
                                          lengths=st["lengths"])
        return y, h_last, dx, dg, dh0
    if op == "norm":
        return seq.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS)
    if op == "norm_train":
        y, mean, rstd = seq.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS, keep=True)
        return (y,) + tuple(seq.layer_norm_grad(st["x"], st["weight"], mean, rstd, st["dy"]))
    if op == "xent":
        return seq.softmax_xent(st["hidden"], st["weight"], st["targets"])
    return seq.softmax_xent_grad(st["hidden"], st["weight"], st["targets"], st["upstream"])


# ------------------------------------------------------------ in 64 bits

def _stepped(a, b, h):
    """All states of h_t = a_t h_{t-1} + b_t, [B, T, D], from h [B, D]: about
    sqrt(T) pieces of the time axis step side by side from zero, then the
    pieces are joined in order."""
    B, T, D = a.shape
    L = max(1, math.isqrt(T))
    P = (T + L - 1) // L
    pad = P * L - T
    if pad:
        a = torch.cat((a, torch.ones((B, pad, D), dtype=a.dtype, device=a.device)), 1)
        b = torch.cat((b, torch.zeros((B, pad, D), dtype=b.dtype, device=b.device)), 1)
    a, b = a.reshape(B, P, L, D), b.reshape(B, P, L, D)
    out, reach = torch.empty_like(a), torch.empty_like(a)
    s, r = torch.zeros_like(a[:, :, 0]), torch.ones_like(a[:, :, 0])
    for i in range(L):
        s = a[:, :, i] * s + b[:, :, i]
        r = r * a[:, :, i]
        out[:, :, i], reach[:, :, i] = s, r
    for p in range(P):
        out[:, p] += reach[:, p] * h[:, None]
        h = out[:, p, L - 1]
    return out.reshape(B, P * L, D)[:, :T]


def _exact_scan(st, train):
    x, g, h0 = st["x"].double(), st["g"].double(), st["h0"].double()
    B, T, D = x.shape
    n = st["lengths"]
    n = torch.full((B,), T, device=x.device) if n is None else n.long()
    on = (torch.arange(T, device=x.device) < n[:, None])[..., None].expand(B, T, D)
    a = 1 / (1 + torch.exp(-g))
    c = 1 / (1 + torch.exp(g))
    keep = a.masked_fill(~on, 1)
    h = _stepped(keep, (c * x).masked_fill(~on, 0), h0)
    y, h_last = h.masked_fill(~on, 0), h[:, -1].clone()
    if not train:
        return y, h_last
    before = torch.cat((h0[:, None], h[:, :-1]), 1)
    dy = st["dy"].double().masked_fill(~on, 0)
    # m_t = a_t l_t is what step t hands to the one before: m_t = a_t m_{t+1} + a_t dy_t
    m = _stepped(keep.flip(1), (keep * dy).flip(1), st["dh_last"].double()).flip(1)
    l = dy + torch.cat((m[:, 1:], st["dh_last"].double()[:, None]), 1)
    dx = (c * l).masked_fill(~on, 0)
    dg = (a * c * (before - x) * l).masked_fill(~on, 0)
    return y, h_last, dx, dg, m[:, 0].clone()


def _exact_norm(st, train):
    x, w = st["x"].double(), st["weight"].double()
    d = x - x.sum(1, keepdim=True) / x.shape[1]
    sigma = torch.sqrt((d * d).sum(1, keepdim=True) / x.shape[1] + EPS)
    y = d / sigma * w + st["bias"].double()
    if not train:
        return y
    dy = st["dy"].double()
    # the derivative of d / sigma, written with d and sigma
    u = dy * w
    dd = u / sigma - d * ((u * d).sum(1, keepdim=True) / x.shape[1]) / sigma ** 3
    dx = dd - dd.sum(1, keepdim=True) / x.shape[1]
    return y, dx, (dy * d / sigma).sum(0), dy.sum(0)


def _exact_xent(st, grad):
    h, W, t = st["hidden"].double(), st["weight"].double(), st["targets"]
    N, V = h.shape[0], W.shape[0]
    loss = torch.zeros(N, dtype=torch.float64, device=h.device)
    lse = torch.zeros_like(loss)
    dh, dW = torch.zeros_like(h), torch.zeros_like(W)
    for r in range(0, N, 1024):  # rows by rows
        hr, tr = h[r:r + 1024], t[r:r + 1024]
        l = hr @ W.t()
        lse[r:r + 1024] = torch.logsumexp(l, 1)
        i = ((tr >= 0) & (tr < V)).nonzero()[:, 0]
        loss[r + i] = lse[r + i] - l[i, tr[i]]
        if grad:
            q = torch.softmax(l, 1)
            q[i, tr[i]] -= 1
            up = torch.zeros(hr.shape[0], dtype=torch.float64, device=h.device)
            up[i] = st["upstream"][r + i].double()
            q *= up[:, None]
            dh[r:r + 1024] = q @ W
            dW += q.t().contiguous() @ hr
    return (dh, dW, loss, lse) if grad else (loss, lse)


def exact(case, seed):
    """The outputs of ``run`` in 64 bits, from the definitions."""
    st = prepare(case, seed)
    op, D = case["op"], case["dim"]
    if op in ("embed", "embed_grad"):
        V = case["vocab"]
        i = ((st["tokens"] >= 0) & (st["tokens"] < V)).nonzero()[:, 0]
        if op == "embed":
            out = torch.zeros((case["tokens"], D), dtype=torch.float64, device="cuda")
            out[i] = st["table"].double()[st["tokens"][i]] * st["scale"]
            return out
        # sums of sorted rows: differences of running sums would lose digits, so add by runs
        t, order = torch.sort(st["tokens"][i])
        ids, counts = torch.unique_consecutive(t, return_counts=True)
        out = torch.zeros((V, D), dtype=torch.float64, device="cuda")
        if ids.numel():
            rows = st["grad_out"][i[order]].double()
            out[ids] = torch.segment_reduce(rows, "sum", lengths=counts, axis=0) * st["scale"]
        return out
    if op in ("scan", "scan_train"):
        return _exact_scan(st, op == "scan_train")
    if op in ("norm", "norm_train"):
        return _exact_norm(st, op == "norm_train")
    return _exact_xent(st, op == "xent_grad")
