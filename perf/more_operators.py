"""The operators of selective models of measurement records, as cases to measure.

A selective model of records runs a short causal convolution and a selective
state space scan over the steps of a record, is trained with clipped gradients
and answers with the most likely records, which a beam search finds.  Every
case is one of these operators, forward or with its gradient:

  scan, scan_train    h_t = exp(d_t A) h_{t-1} + d_t x_t B_t, d_t = softplus(dt_t + bias),
                      y_t = (C_t . h_t + skip x_t) silu(z_t)
  conv, conv_train    y_t = silu(bias + sum_k weight_k x_{t-K+1+k})
  clip                norm of all gradients of a model, gradients cut to a largest norm
  beam                the best continuations of the beams over the vocabulary
  reorder             the beams' states, gathered by the beams they continue

Where ``own`` is false ``run`` computes them in their plain form, with
elementary torch operations in 32 bits (the selection and the norm in 64);
where it is true it calls the framework.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
NO_ID = -1


def listed():
    return [
        # one step of 1024 records that are being extended: a call for a single token, state read and written
        {"name": "scan_step_b1024_bf16", "op": "scan", "type": "bf16", "batch": 1024, "steps": 1, "dim": 512,
         "state": 16, "ragged": False},
        # one long record (repeated measurement of one device): a long axis, little to do side by side; odd width
        {"name": "scan_b1_t100001_f32", "op": "scan", "type": "f32", "batch": 1, "steps": 100001, "dim": 331,
         "state": 16, "ragged": False},
        # the largest: a training step over records of different lengths, empty ones among them
        {"name": "scan_train_b8_t4099_bf16", "op": "scan_train", "type": "bf16", "batch": 8, "steps": 4099,
         "dim": 1024, "state": 16, "ragged": True},
        # advancing 64 records by one step: all latency
        {"name": "conv_step_b64_f32", "op": "conv", "type": "f32", "batch": 64, "steps": 1, "dim": 200, "taps": 4,
         "ragged": False},
        # a training step's convolution over records of different lengths
        {"name": "conv_train_b24_t4099_bf16", "op": "conv_train", "type": "bf16", "batch": 24, "steps": 4099,
         "dim": 1024, "taps": 4, "ragged": True},
        # an odd width and few records
        {"name": "conv_train_b3_t20011_f16", "op": "conv_train", "type": "f16", "batch": 3, "steps": 20011, "dim": 331,
         "taps": 3, "ragged": False},
        # the gradients of a one-layer model of 4 qubits' records: all latency
        {"name": "clip_n4_f32", "op": "clip", "type": "f32", "qubits": 4, "width": 64, "layers": 1, "over": True},
        # those of six layers over the bitstrings of 16 qubits, in 16 bits with a loss scale, to 32 bits
        {"name": "clip_n16_l6_f16", "op": "clip", "type": "f16", "qubits": 16, "width": 1024, "layers": 6,
         "over": True},
        # the next bitstring of 16 records of 4 qubits with 4 beams each: all latency
        {"name": "beam_n4_b16_w4_f32", "op": "beam", "type": "f32", "records": 16, "beams": 4, "vocab": 17,
         "ends": False, "masked": False},
        # 64 records with 8 beams each over all bitstrings of 16 qubits; some records have ended, some words cannot follow
        {"name": "beam_n16_b64_w8_bf16", "op": "beam", "type": "bf16", "records": 64, "beams": 8, "vocab": 65537,
         "ends": True, "masked": True},
        # the states of those 16 records' beams: one layer
        {"name": "reorder_b16_w4_l1", "op": "reorder", "type": "bf16", "records": 16, "beams": 4, "dim": 64,
         "state": 16, "taps": 4, "layers": 1},
        # the states of 64 records with 8 beams in twelve layers
        {"name": "reorder_b64_w8_l12", "op": "reorder", "type": "bf16", "records": 64, "beams": 8, "dim": 1024,
         "state": 16, "taps": 4, "layers": 12},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A further case: operator, direction, type and sizes over the ranges
    that the listed ones stand for, at most the largest listed one's work."""
    most = {k: max(work(c)[k] for c in listed()) for k in ("flops", "bytes")}
    while True:
        op = rng.choice(("scan", "scan_train", "scan", "scan_train", "conv", "conv_train", "clip", "beam", "reorder"))
        c = {"op": op, "type": rng.choice(("f32", "bf16", "f16"))}
        if op in ("scan", "scan_train", "conv", "conv_train"):
            c.update(batch=_log(rng, 1, 4096), steps=rng.choice((1, _log(rng, 2, 131072), _log(rng, 2, 131072))),
                     dim=_log(rng, 16, 2048), ragged=rng.random() < 0.5)
            if op in ("scan", "scan_train"):
                c.update(state=rng.choice((16, 16, rng.randint(1, 64))))
            else:
                c.update(taps=rng.choice((4, rng.randint(2, 8))))
        elif op == "clip":
            c.update(qubits=rng.randint(2, 16), width=_log(rng, 16, 1024), layers=rng.randint(1, 6),
                     over=rng.random() < 0.7)
        elif op == "beam":
            c.update(records=_log(rng, 1, 2048), beams=_log(rng, 1, 32), vocab=(1 << rng.randint(5, 18)) + 1,
                     ends=rng.random() < 0.5, masked=rng.random() < 0.5)
        else:
            c.update(records=_log(rng, 1, 1024), beams=_log(rng, 1, 32), dim=_log(rng, 16, 2048),
                     state=rng.choice((16, rng.randint(1, 64))), taps=rng.randint(2, 8), layers=_log(rng, 1, 24))
        w = work(c)
        # the plain scan keeps some twelve arrays of all states in 32 bits: 2^29 of them are 2 GB
        states = c.get("batch", 0) * c.get("steps", 0) * c.get("dim", 0) * c.get("state", 1)
        chosen = c.get("records", 0) * c.get("beams", 0) * c.get("vocab", 0)
        if w["flops"] <= most["flops"] and w["bytes"] <= most["bytes"] and states <= 1 << 29 and chosen <= 1 << 26:
            return c


def _size(case):
    return 4 if case["type"] == "f32" else 2


def _shapes(case):
    """The gradients of a selective model's parameters: (shape, whether in the
    case's type; the scan's own parameters are held in 32 bits)."""
    V, W, S = (1 << case["qubits"]) + 1, case["width"], 16
    out = [((V, W), True), ((V, W), True)]  # table, readout
    for _ in range(case["layers"]):
        out += [((W, 2 * W + 33), True), ((W, W), True), ((4, W), True), ((W,), True),  # products, convolution
                ((W, S), False), ((W,), False), ((W,), False), ((W,), True), ((W,), True)]  # scan, norm
    return out


def work(case):
    """Each input read once and each output written once; products, sums and
    exponentials of the formulas."""
    s, op = _size(case), case["op"]
    if op in ("scan", "scan_train", "conv", "conv_train"):
        B, T, D = case["batch"], case["steps"], case["dim"]
        # records of different lengths fill about half of the steps; outputs are written whole
        fill = 0.5 if case["ragged"] else 1.0
        n = B * T * D
        if op in ("scan", "scan_train"):
            S = case["state"]
            state, params = 4 * B * D * S, 4 * D * (S + 2)
            if op == "scan":  # x, dt, z, B, C; y
                return {"bytes": int((n * (3 * fill + 1) + 2 * fill * B * T * S) * s) + 2 * state + params,
                        "flops": int(n * fill * (7 * S + 12))}
            # dy too; y, dx, ddt, dz, dB, dC
            return {"bytes": int((n * (4 * fill + 4) + (2 * fill + 2) * B * T * S) * s) + 4 * state + 2 * params,
                    "flops": int(n * fill * (20 * S + 40))}
        K = case["taps"]
        state, params = B * (K - 1) * D * s, (K + 1) * D * s
        if op == "conv":
            return {"bytes": int(n * s * (fill + 1)) + 2 * state + params, "flops": int(n * fill * (2 * K + 4))}
        return {"bytes": int(n * s * (2 * fill + 2)) + 4 * state + 2 * params, "flops": int(n * fill * (8 * K + 16))}
    if op == "clip":
        n = sum(math.prod(shape) for shape, _ in _shapes(case))
        read = sum(math.prod(shape) * (s if typed else 4) for shape, typed in _shapes(case))
        return {"bytes": read + 4 * n, "flops": 3 * n}
    R, W = case["records"], case["beams"]
    if op == "beam":
        return {"bytes": R * W * (case["vocab"] * s + 28), "flops": 4 * R * W * case["vocab"]}
    D, layers = case["dim"], case["layers"]
    row = layers * D * (4 * case["state"] + (case["taps"] - 1) * s)
    return {"bytes": 2 * R * W * row, "flops": R * W}


# ------------------------------------------------------------------- inputs

def _normal(gen, shape, dtype, scale=1.0, shift=0.0):
    return (torch.randn(shape, device=gen.device, generator=gen) * scale + shift).to(dtype)


def _lengths(gen, case):
    if not case["ragged"]:
        return None
    n = torch.randint(0, case["steps"] + 1, (case["batch"],), device="cuda", generator=gen, dtype=torch.int32)
    n[0] = 0
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dt = case["op"], TYPES[case["type"]]
    st = {"case": case}
    if op in ("scan", "scan_train"):
        B, T, D, S = case["batch"], case["steps"], case["dim"], case["state"]
        # parts of one array, as a model's product or table gives them
        parts = _normal(gen, (B, T, 3 * D + 2 * S), dt)
        st["x"], st["dt"], st["z"] = parts[..., :D], parts[..., D:2 * D], parts[..., 2 * D:3 * D]
        st["B"], st["C"] = parts[..., 3 * D:3 * D + S], parts[..., 3 * D + S:]
        # memories of a step to a thousand: steps of 0.001 to 0.1, decays of 1 to S
        step = torch.exp(torch.rand(D, device="cuda", generator=gen) * math.log(100.0) + math.log(1e-3))
        st["dt_bias"] = torch.log(torch.expm1(step))
        decay = torch.arange(1, S + 1, device="cuda", dtype=torch.float32)
        st["A"] = -decay * torch.exp(_normal(gen, (D, S), torch.float32, 0.1))
        st["skip"] = _normal(gen, (D,), torch.float32, 0.1, 1.0)
        st["h0"] = _normal(gen, (B, D, S), torch.float32, 0.3)
        st["lengths"] = _lengths(gen, case)
        if op == "scan_train":
            st["dy"] = _normal(gen, (B, T, D), dt)
            st["dh_last"] = _normal(gen, (B, D, S), torch.float32)
    elif op in ("conv", "conv_train"):
        B, T, D, K = case["batch"], case["steps"], case["dim"], case["taps"]
        st["x"] = _normal(gen, (B, T, D), dt)
        st["weight"] = _normal(gen, (K, D), dt, 1 / math.sqrt(K))
        st["bias"] = _normal(gen, (D,), dt, 0.1)
        st["state"] = _normal(gen, (B, K - 1, D), dt)
        st["lengths"] = _lengths(gen, case)
        if op == "conv_train":
            st["dy"] = _normal(gen, (B, T, D), dt)
            st["dlast"] = _normal(gen, (B, K - 1, D), dt)
    elif op == "clip":
        # 16 bits: the gradients of a loss times 1024
        st["scale"] = 1.0 if case["type"] == "f32" else 1.0 / 1024
        shapes = _shapes(case)
        count = sum(math.prod(shape) for shape, _ in shapes)
        size = (4.0 if case["over"] else 0.5) / math.sqrt(count) / st["scale"]
        st["grads"] = [_normal(gen, shape, dt if typed else torch.float32, size) for shape, typed in shapes]
        # what the optimiser reads is kept from step to step
        st["out"] = [torch.empty(shape, device="cuda") for shape, _ in shapes]
        st["max_norm"] = 1.0
    elif op == "beam":
        R, W, V = case["records"], case["beams"], case["vocab"]
        st["logits"] = _normal(gen, (R, W, V), dt, 2.0)
        if case["masked"]:  # words that cannot follow, a quarter of them
            st["logits"].masked_fill_(torch.rand((1, 1, V), device="cuda", generator=gen) < 0.25, -math.inf)
            st["logits"][..., 0] = 0.5
        st["scores"] = _normal(gen, (R, W), torch.float32, 1.0, -20.0)
        st["scores"][0, 1:] = -math.inf  # a record that begins: one beam
        st["last"], st["end"] = None, NO_ID
        if case["ends"]:
            st["end"] = V - 1
            st["last"] = torch.randint(0, V - 1, (R, W), device="cuda", generator=gen)
            st["last"][torch.rand((R, W), device="cuda", generator=gen) < 0.2] = V - 1
    else:
        R, W, D = case["records"], case["beams"], case["dim"]
        st["states"] = []
        for _ in range(case["layers"]):
            st["states"] += [_normal(gen, (R, W, D, case["state"]), torch.float32),
                             _normal(gen, (R, W, case["taps"] - 1, D), dt)]
        st["parents"] = torch.randint(0, W, (R, W), device="cuda", generator=gen, dtype=torch.int32)
        # the states of the step before, written over
        st["out"] = [torch.empty_like(t) for t in st["states"]]
    return st


# -------------------------------------------------------------- plain forms

def _on(lengths, B, T, device):
    if lengths is None:
        return None
    return torch.arange(T, device=device)[None, :] < lengths[:, None]


def _doubling(a, b):
    """h_t = a_t h_{t-1} + b_t along dim 1 from h = 0, by doubling the span
    each step covers."""
    T, d = a.shape[1], 1
    while d < T:
        b = torch.cat((b[:, :d], a[:, d:] * b[:, :-d] + b[:, d:]), 1)
        if 2 * d < T:
            a = torch.cat((a[:, :d], a[:, d:] * a[:, :-d]), 1)
        d *= 2
    return b


def _plain_scan(st, train):
    x, z = st["x"].float(), st["z"].float()
    Bm, Cm, A, h0 = st["B"].float(), st["C"].float(), st["A"], st["h0"]
    v = st["dt"].float() + st["dt_bias"]
    e = torch.exp(-v.abs())
    delta = v.clamp(min=0) + torch.log1p(e)
    B, T, D = x.shape
    on, zero = _on(st["lengths"], B, T, x.device), torch.zeros((), device=x.device)
    if on is not None:  # steps past the end carry the state on
        on = on[..., None]
        x, delta, z = torch.where(on, x, zero), torch.where(on, delta, zero), torch.where(on, z, zero)
        Bm, Cm = torch.where(on, Bm, zero), torch.where(on, Cm, zero)
    a = torch.exp(delta[..., None] * A)
    b = (delta * x)[..., None] * Bm[:, :, None]
    b[:, 0] += a[:, 0] * h0
    h = _doubling(a, b)
    del b
    p = (h * Cm[:, :, None]).sum(-1) + st["skip"] * x
    sz = 1 / (1 + torch.exp(-z))
    gate = z * sz
    dtype = st["x"].dtype
    y = (p * gate).to(dtype)
    h_last = h[:, -1].clone()
    if not train:
        return y, h_last
    dy = st["dy"].float()
    if on is not None:
        dy = torch.where(on, dy, zero)
    q = dy * gate
    dz = dy * p * (sz + gate * (1 - sz))
    dC = (h * q[..., None]).sum(2)
    # l_t = q_t C_t + a_{t+1} l_{t+1}, from the last step back
    l = q[..., None] * Cm[:, :, None]
    l[:, -1] += st["dh_last"]
    nxt = torch.cat((a[:, 1:], torch.ones_like(a[:, :1])), 1)
    l = _doubling(nxt.flip(1), l.flip(1)).flip(1)
    del nxt
    bl = (l * Bm[:, :, None]).sum(-1)
    dx = delta * bl + st["skip"] * q
    dB = (l * (delta * x)[..., None]).sum(2)
    dh0 = a[:, 0] * l[:, 0]
    l *= a
    l *= torch.cat((h0[:, None], h[:, :-1]), 1)
    dA = (l * delta[..., None]).sum((0, 1))
    ddelta = (l * A).sum(-1) + x * bl
    ddt = ddelta * torch.where(v >= 0, 1 / (1 + e), e / (1 + e))
    if on is not None:
        ddt = torch.where(on, ddt, zero)
    return (y, h_last, dx.to(dtype), ddt.to(dtype), dA, dB.to(dtype), dC.to(dtype), (q * x).sum((0, 1)), dz.to(dtype),
            ddt.sum((0, 1)), dh0)


def _plain_conv(st, train):
    x, w, bias = st["x"].float(), st["weight"].float(), st["bias"].float()
    B, T, D = x.shape
    K, dtype = w.shape[0], st["x"].dtype
    on, zero = _on(st["lengths"], B, T, x.device), torch.zeros((), device=x.device)
    if on is not None:
        on = on[..., None]
        x = torch.where(on, x, zero)
    # the inputs before the record, then its own
    xs = torch.cat((st["state"].float(), x), 1)
    u = bias + sum(w[k] * xs[:, k:k + T] for k in range(K))
    sg = 1 / (1 + torch.exp(-u))
    y = u * sg
    if on is not None:
        y = torch.where(on, y, zero)
    n = torch.full((B,), T, device=x.device) if st["lengths"] is None else st["lengths"].long()
    at = (n[:, None] + torch.arange(K - 1, device=x.device))[..., None].expand(B, K - 1, D)
    last = xs.gather(1, at).to(dtype)
    y = y.to(dtype)
    if not train:
        return y, last
    g = st["dy"].float() * (sg * (1 + u * (1 - sg)))
    if on is not None:
        g = torch.where(on, g, zero)
    dxs = torch.zeros_like(xs)
    dxs.scatter_(1, at, st["dlast"].float())
    for k in range(K):
        dxs[:, k:k + T] += w[k] * g
    dw = torch.stack([(g * xs[:, k:k + T]).sum((0, 1)) for k in range(K)])
    dx = dxs[:, K - 1:]
    if on is not None:
        dx = torch.where(on, dx, zero)
    return y, last, dx.to(dtype), dw.to(dtype), g.sum((0, 1)).to(dtype), dxs[:, :K - 1].to(dtype)


def _plain_clip(st):
    total = sum((g.double() ** 2).sum() for g in st["grads"])
    norm = total.sqrt() * st["scale"]
    coefficient = st["scale"] * torch.where(norm <= st["max_norm"], torch.ones_like(norm), st["max_norm"] / norm)
    for g, o in zip(st["grads"], st["out"]):
        o.copy_(g.float() * coefficient.float())
    return norm.float(), st["out"]


def _candidates(scores, logits, last, end):
    """The score of every continuation [R, W * V] in 64 bits, -inf where there is none."""
    z = logits.double()
    top = z.max(-1, keepdim=True).values
    lse = (z - top).exp().sum(-1, keepdim=True).log() + top
    s = scores.double()[..., None]
    cand = s + (z - lse)
    none = torch.full((), -math.inf, dtype=torch.float64, device=z.device)
    if last is not None:  # a beam that has ended goes on as it is
        ended = (last == end)[..., None]
        word = torch.arange(z.shape[-1], device=z.device)
        cand = torch.where(ended, torch.where(word == end, s, none), cand)
    cand = torch.where(cand < math.inf, cand, none)
    return cand.flatten(1)


def _plain_beam(st):
    W, V = st["logits"].shape[1:]
    best, at = torch.sort(_candidates(st["scores"], st["logits"], st["last"], st["end"]), dim=1, descending=True,
                          stable=True)
    best, at = best[:, :W], at[:, :W]
    return best.float(), (at // V).int(), at % V


def _plain_reorder(st):
    row = torch.arange(st["parents"].shape[0], device=st["parents"].device)[:, None]
    at = st["parents"].long()
    for t, o in zip(st["states"], st["out"]):
        o.copy_(t[row, at])
    return st["out"]


def run(st):
    if own:
        return _run_own(st)
    op = st["case"]["op"]
    if op in ("scan", "scan_train"):
        return _plain_scan(st, op == "scan_train")
    if op in ("conv", "conv_train"):
        return _plain_conv(st, op == "conv_train")
    return {"clip": _plain_clip, "beam": _plain_beam, "reorder": _plain_reorder}[op](st)


def _run_own(st):
    from paper_2003_02989_amd import model
    op = st["case"]["op"]
    if op in ("scan", "scan_train"):
        args = (st["x"], st["dt"], st["A"], st["B"], st["C"])
        more = {"skip": st["skip"], "z": st["z"], "dt_bias": st["dt_bias"], "lengths": st["lengths"]}
        if op == "scan":
            return model.selective_scan(*args, h0=st["h0"], **more)
        y, h_last, states = model.selective_scan(*args, h0=st["h0"], keep=True, **more)
        g = model.selective_scan_grad(*args, states, st["dy"], dh_last=st["dh_last"], **more)
        return (y, h_last, g.dx, g.ddt, g.dA, g.dB, g.dC, g.dskip, g.dz, g.ddt_bias, g.dh0)
    if op in ("conv", "conv_train"):
        out = model.causal_conv(st["x"], st["weight"], bias=st["bias"], state=st["state"], lengths=st["lengths"])
        if op == "conv":
            return out
        return out + tuple(model.causal_conv_grad(st["x"], st["weight"], st["dy"], bias=st["bias"], state=st["state"],
                                                  dlast=st["dlast"], lengths=st["lengths"]))
    if op == "clip":
        return model.clip_grad_norm(st["grads"], st["max_norm"], scale=st["scale"], out=st["out"])
    if op == "beam":
        return model.beam_select(st["logits"], st["scores"], last=st["last"], end=st["end"])
    return model.beam_reorder(st["states"], st["parents"], out=st["out"])


# ------------------------------------------------------------ in 64 bits

def _stepped(a, b, h):
    """All states of h_t = a_t h_{t-1} + b_t, [B, T, ...], from h [B, ...]:
    about sqrt(T) pieces of the time axis step side by side from zero, then the
    pieces are joined in order."""
    B, T = a.shape[:2]
    rest = a.shape[2:]
    L = max(1, math.isqrt(T))
    P = (T + L - 1) // L
    pad = P * L - T
    if pad:
        a = torch.cat((a, a.new_ones((B, pad) + rest)), 1)
        b = torch.cat((b, b.new_zeros((B, pad) + rest)), 1)
    a, b = a.reshape((B, P, L) + rest), b.reshape((B, P, L) + rest).clone()
    s, r = torch.zeros_like(a[:, :, 0]), torch.ones_like(a[:, :, 0])
    for i in range(L):
        s = a[:, :, i] * s + b[:, :, i]
        b[:, :, i] = s
    for p in range(P):  # the piece before it reaches every step of this one
        r = torch.cumprod(a[:, p], 1)
        b[:, p] += r * h[:, None]
        h = b[:, p, L - 1]
    return b.reshape((B, P * L) + rest)[:, :T]


def _exact_scan(st, train):
    x, dt, z, Bm, Cm = (st[k].double() for k in ("x", "dt", "z", "B", "C"))
    A, skip, h0 = st["A"].double(), st["skip"].double(), st["h0"].double()
    B, T, D = x.shape
    n = st["lengths"]
    n = torch.full((B,), T, device=x.device) if n is None else n.long()
    off = ~(torch.arange(T, device=x.device) < n[:, None])[..., None]
    v = dt + st["dt_bias"].double()
    delta = torch.logaddexp(v, torch.zeros_like(v)).masked_fill(off, 0)
    a = torch.exp(torch.einsum("btd,ds->btds", delta, A))
    h = _stepped(a, torch.einsum("btd,bts->btds", delta * x, Bm).masked_fill(off[..., None], 0), h0)
    gate = z * torch.sigmoid(z)
    p = torch.matmul(h, Cm[..., None])[..., 0] + skip * x
    y, h_last = (p * gate).masked_fill(off, 0), h[:, -1].clone()
    if not train:
        return y, h_last
    dy = st["dy"].double().masked_fill(off, 0)
    s = torch.sigmoid(z)
    dz = (dy * p * s * (1 + z * (1 - s))).masked_fill(off, 0)
    q = (dy * gate).masked_fill(off, 0)
    dC = torch.matmul(q[:, :, None], h)[:, :, 0]
    # m_t = a_t l_t is what step t hands to the one before: m_t = a_t m_{t+1} + a_t q_t C_t
    qc = torch.einsum("btd,bts->btds", q, Cm.masked_fill(off, 0))
    m = _stepped(a.flip(1), (a * qc).flip(1), st["dh_last"].double()).flip(1)
    del a
    l = qc
    l[:, :-1] += m[:, 1:]
    l[:, -1] += st["dh_last"].double()
    dh0 = m[:, 0].clone()
    bl = torch.matmul(l, Bm[..., None])[..., 0]
    dB = torch.matmul((delta * x)[:, :, None], l)[:, :, 0].masked_fill(off, 0)
    dx = (delta * bl + skip * q).masked_fill(off, 0)
    del l, qc
    m[:, 1:] *= h[:, :-1]
    m[:, 0] *= h0
    m.masked_fill_(off[..., None], 0)
    dA = torch.einsum("btds,btd->ds", m, delta)
    ddt = ((torch.einsum("btds,ds->btd", m, A) + x * bl) * torch.sigmoid(v)).masked_fill(off, 0)
    return (y, h_last, dx, ddt, dA, dB, dC, (q * x).masked_fill(off, 0).sum((0, 1)), dz, ddt.sum((0, 1)), dh0)


def _exact_conv(st, train):
    x, w, bias, state = (st[k].double() for k in ("x", "weight", "bias", "state"))
    B, T, D = x.shape
    K = w.shape[0]
    n = st["lengths"]
    n = [T] * B if n is None else n.tolist()
    out = [torch.zeros_like(x), torch.zeros_like(state), torch.zeros_like(x), torch.zeros_like(w),
           torch.zeros_like(bias), torch.zeros_like(state)]
    for b in range(B):  # record by record, as long as each one is
        row = torch.cat((state[b], x[b, :n[b]]))
        out[1][b] = row[n[b]:]
        if not n[b]:
            out[5][b] = st["dlast"][b].double() if train else 0
            continue
        win = row.unfold(0, K, 1)  # [steps, D, K]
        u = torch.einsum("tdk,kd->td", win, w) + bias
        s = torch.sigmoid(u)
        out[0][b, :n[b]] = u * s
        if train:
            g = st["dy"][b, :n[b]].double() * (s + u * s * (1 - s))
            back = torch.zeros_like(row)
            back[n[b]:] = st["dlast"][b].double()
            for k in range(K):
                back[k:k + n[b]] += w[k] * g
            out[2][b, :n[b]] = back[K - 1:]
            out[5][b] = back[:K - 1]
            out[3] += torch.einsum("tdk,td->kd", win, g)
            out[4] += g.sum(0)
    return tuple(out) if train else tuple(out[:2])


def _exact_beam(st):
    """The best one, taken out, and again."""
    z, W, V = st["logits"].double(), st["logits"].shape[1], st["logits"].shape[2]
    total = st["scores"].double()[..., None] + torch.log_softmax(z, -1)
    if st["last"] is not None:
        over = st["last"] == st["end"]
        total[over] = -math.inf
        total[..., st["end"]] = torch.where(over, st["scores"].double(), total[..., st["end"]])
    flat = torch.nan_to_num(total.flatten(1), nan=-math.inf, neginf=-math.inf)
    rank = torch.arange(W * V, device=z.device).expand_as(flat)
    left = torch.ones_like(flat, dtype=torch.bool)
    scores, picks = [], []
    for _ in range(W):
        best = flat.masked_fill(~left, -math.inf).amax(1, keepdim=True)
        at = rank.masked_fill(~(left & (flat == best)), W * V).amin(1, keepdim=True)
        left.scatter_(1, at, False)
        scores.append(best)
        picks.append(at)
    at = torch.cat(picks, 1)
    return torch.cat(scores, 1), (at // V).int(), at % V


def exact(case, seed):
    """The outputs of ``run`` in 64 bits, from the definitions."""
    st = prepare(case, seed)
    op = case["op"]
    if op in ("scan", "scan_train"):
        return _exact_scan(st, op == "scan_train")
    if op in ("conv", "conv_train"):
        return _exact_conv(st, op == "conv_train")
    if op == "clip":
        flat = torch.cat([g.flatten().double() for g in st["grads"]]) * st["scale"]
        norm = torch.linalg.vector_norm(flat)
        c = min(1.0, st["max_norm"] / float(norm))
        return norm, [g.double() * (st["scale"] * c) for g in st["grads"]]
    if op == "beam":
        return _exact_beam(st)
    R, W = st["parents"].shape
    at = (st["parents"].long() + W * torch.arange(R, device="cuda")[:, None]).flatten()
    return [t.flatten(0, 1).index_select(0, at).view(t.shape).double() for t in st["states"]]
