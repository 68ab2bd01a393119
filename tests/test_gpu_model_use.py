"""The operators of selective models as programs use them: streams, captured
graphs, layouts, values and sizes at their ends, the same bits from call to call."""
import numpy as np
import pytest
import torch

from paper_2003_02989_amd import model

pytestmark = pytest.mark.gpu


def scan_set(B=2, T=700, D=70, S=9, dtype=torch.bfloat16, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def n(*shape, dt=dtype):
        return torch.randn(shape, device="cuda", generator=gen).to(dt)
    f = torch.float32
    return {"x": n(B, T, D), "dt": n(B, T, D) - 2, "z": n(B, T, D), "B": n(B, T, S), "C": n(B, T, S),
            "A": -torch.exp(n(D, S, dt=f)), "skip": n(D, dt=f), "dt_bias": n(D, dt=f), "h0": n(B, D, S, dt=f),
            "dy": n(B, T, D), "dh": n(B, D, S, dt=f),
            "w": n(4, D), "bias": n(D), "state": n(B, 3, D), "dlast": n(B, 3, D),
            "logits": n(6, 4, 5000), "scores": n(6, 4, dt=f), "grads": [n(400, 300), n(70, dt=f), n(33, 7)],
            "parents": torch.randint(0, 4, (6, 4), device="cuda", generator=gen, dtype=torch.int32),
            "states": [n(6, 4, 33, 7), n(6, 4, 5000)]}


def everything(s, **kw):
    """Each operator once, all outputs."""
    args = (s["x"], s["dt"], s["A"], s["B"], s["C"])
    more = dict(skip=s["skip"], z=s["z"], dt_bias=s["dt_bias"])
    y, h, states = model.selective_scan(*args, h0=s["h0"], keep=True, **more, **kw)
    g = model.selective_scan_grad(*args, states, s["dy"], dh_last=s["dh"], **more, **kw)
    one = model.selective_scan(*(t[:, :1] for t in args[:2]), args[2], *(t[:, :1] for t in args[3:]), h0=s["h0"], **kw)
    c = model.causal_conv(s["x"], s["w"], bias=s["bias"], state=s["state"], **kw)
    cg = model.causal_conv_grad(s["x"], s["w"], s["dy"], bias=s["bias"], state=s["state"], dlast=s["dlast"], **kw)
    norm, outs = model.clip_grad_norm(s["grads"], 1.0, out=[torch.empty_like(t) for t in s["grads"]], **kw)
    picks = model.beam_select(s["logits"], s["scores"], **kw)
    small = model.beam_select(s["logits"][..., :100], s["scores"], **kw)
    moved = model.beam_reorder(s["states"], s["parents"], **kw)
    return [y, h, *g, *one, *c, *cg, norm, *outs, *picks, *small, *moved]


def same(a, b):
    assert len(a) == len(b)
    return all(torch.equal(p, q) for p, q in zip(a, b))


def test_every_call_gives_the_same_bits():
    s = scan_set()
    want = everything(s)
    assert all(torch.isfinite(t.float()).all() for t in want)
    for _ in range(4):
        assert same(everything(s), want)


def test_other_streams():
    s = scan_set(seed=1)
    want = everything(s)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    got = everything(s, stream=side)
    with torch.cuda.stream(other):  # both at once, each with workspaces of its own
        again = everything(s)
    side.synchronize()
    other.synchronize()
    assert same(got, want) and same(again, want)


def test_graph_replays():
    """Two graphs captured one after the other, replayed in turns with other inputs
    and eager calls between."""
    kept = [scan_set(seed=2), scan_set(seed=3)]
    graphs, outs = [], []
    for s in kept:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            everything(s)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = everything(s)
        graphs.append(g)
        outs.append(out)
    for turn in range(4):
        for s in kept:
            fresh = scan_set(seed=10 + turn)
            for k, v in s.items():
                for a, b in zip(v, fresh[k]) if isinstance(v, list) else [(v, fresh[k])]:
                    a.copy_(b)
        for g in graphs:
            g.replay()
        want = everything(kept[0])
        torch.cuda.synchronize()
        for out in outs:
            assert same(out, want), turn


@pytest.mark.parametrize("T", [1, 5, 900])
def test_states_advance_in_place(T):
    s = scan_set(T=T, seed=4)
    args = (s["x"], s["dt"], s["A"], s["B"], s["C"])
    y, h = model.selective_scan(*args, h0=s["h0"])
    kept = s["h0"].clone()
    y2, h2 = model.selective_scan(*args, h0=kept, h_last=kept)
    assert h2 is kept and torch.equal(h, kept) and torch.equal(y, y2)
    c, last = model.causal_conv(s["x"], s["w"], state=s["state"])
    kept = s["state"].clone()
    c2, _ = model.causal_conv(s["x"], s["w"], state=kept, last=kept)
    assert torch.equal(kept, last) and torch.equal(c, c2)


def test_steps_outermost_and_broadcast_inputs():
    """[T, B, D] arrays as [B, T, D] views; B and C shared by all records; outputs in
    views of one array."""
    s = scan_set(B=3, T=40, seed=5)
    turned = {k: s[k].transpose(0, 1).contiguous().transpose(0, 1) for k in ("x", "dt", "z", "B", "C", "dy")}
    for k in ("B", "C"):
        turned[k] = turned[k][:1].expand(3, -1, -1)
        s[k] = s[k][:1].repeat(3, 1, 1)
    assert same(everything(s)[:11], everything({**s, **turned})[:11])
    D, S = s["x"].shape[2], s["A"].shape[1]
    de = torch.full((3, 40, 3 * D + 2 * S), 7.0, dtype=torch.bfloat16, device="cuda")
    dx, ddt, dz, dB, dC = de.split((D, D, D, S, S), -1)
    args = (s["x"], s["dt"], s["A"], s["B"], s["C"])
    _, _, states = model.selective_scan(*args, z=s["z"], keep=True)
    want = model.selective_scan_grad(*args, states, s["dy"], z=s["z"])
    model.selective_scan_grad(*args, states, s["dy"], z=s["z"], dx=dx, ddt=ddt, dB=dB, dC=dC, dz=dz)
    assert same([dx, ddt, dB, dC, dz], [want.dx, want.ddt, want.dB, want.dC, want.dz])


@pytest.mark.parametrize("T", [1, 40, 1500])
def test_decays_and_steps_at_their_ends(T):
    """Decays of infinity forget at once, of zero nothing; steps of infinite size and
    of none at all."""
    B, D, S = 1, 8, 2
    one = torch.ones((B, T, S), device="cuda")
    x = torch.randn((B, T, D), device="cuda")
    dt = torch.zeros((B, T, D), device="cuda")
    A = torch.zeros((D, S), device="cuda")
    A[:4] = float("-inf")
    h0 = torch.randn((B, D, S), device="cuda")
    y, h = model.selective_scan(x, dt, A, one, one, h0=h0)
    d = np.log(2)
    want = torch.cumsum(x.double(), 1) * d + h0[:, None, :, 0].double()
    keep = want * 0 + x.double() * d
    assert torch.allclose(h[0, :4, 0].double(), keep[0, -1, :4], rtol=1e-5)
    # a sum of up to 1500 terms in fp32: 1500 units of the sum of magnitudes
    most = T * 6e-8 * float(x.abs().sum(1).max())
    assert torch.allclose(h[0, 4:, 0].double(), want[0, -1, 4:], rtol=1e-5, atol=most + 1e-6)
    both = 2 * torch.cumsum(x.double(), 1) * d + h0.double().sum(-1)[:, None]  # y: the sum of both states
    assert torch.allclose(y[..., 4:].double(), both[..., 4:], rtol=1e-5, atol=2 * most + 2e-6)
    dt[:] = float("-inf")  # no step at all: the states stay
    y, h = model.selective_scan(x, dt, torch.full_like(A, -1.0), one, one, h0=h0)
    assert torch.equal(h, h0) and torch.allclose(y, h0.sum(-1)[:, None].expand_as(y), rtol=1e-6)


def test_bad_values_stay_in_their_channel_and_record():
    s = scan_set(B=3, T=300, dtype=torch.float32, seed=6)
    want = everything(s)
    s["x"][1, 100, 5] = float("nan")
    got = everything(s)
    ok = torch.ones((3, 70), dtype=torch.bool)
    ok[1, 5] = False
    for a, b in zip(got[:2], want[:2]):  # y and h_last
        a, b = (a.transpose(1, 2), b.transpose(1, 2)) if a.shape[1] == 300 else (a, b)
        assert torch.equal(a[ok], b[ok]) and torch.isnan(a[1, 5]).any()
    assert torch.equal(got[0][1, :100, 5], want[0][1, :100, 5])
    c, d = model.causal_conv(s["x"], s["w"].float(), silu=False)[0], s["x"][1, 104:, 5]
    assert torch.isnan(c[1, 100:104, 5]).all() and torch.isfinite(c[1, 104:, 5]).all() and torch.isfinite(d).all()


FAR = (1 << 31) + 4096


def test_strides_past_32_bits():
    """Records, rows and tensors that lie more than 2^31 elements apart."""
    dtype, T, D, S = torch.bfloat16, 20, 40, 6
    room = torch.empty(FAR + 8 * T * D, dtype=dtype, device="cuda")
    room2 = torch.empty_like(room)
    s = scan_set(T=T, D=D, S=S, dtype=dtype, seed=7)

    def far(t, at, where):
        v = where[at:].as_strided(t.shape, (FAR, t.shape[2], 1))
        return v.copy_(t)
    names = ("x", "dt", "z", "B", "C", "dy")
    apart = {k: far(s[k], i * T * D, room) for i, k in enumerate(names)}
    y = room2.as_strided((2, T, D), (FAR, D, 1))
    dx = room2[T * D:].as_strided((2, T, D), (FAR, D, 1))
    more = dict(skip=s["skip"], dt_bias=s["dt_bias"])
    wy, wh, wstates = model.selective_scan(s["x"], s["dt"], s["A"], s["B"], s["C"], z=s["z"], keep=True, **more)
    a = apart
    _, h, states = model.selective_scan(a["x"], a["dt"], s["A"], a["B"], a["C"], z=a["z"], keep=True, y=y, **more)
    assert same([y, h, states], [wy, wh, wstates])
    wg = model.selective_scan_grad(s["x"], s["dt"], s["A"], s["B"], s["C"], states, s["dy"], z=s["z"], **more)
    g = model.selective_scan_grad(a["x"], a["dt"], s["A"], a["B"], a["C"], states, a["dy"], z=a["z"], dx=dx, **more)
    assert same(list(g), list(wg))
    wc, _ = model.causal_conv(s["x"], s["w"])
    model.causal_conv(a["x"], s["w"], y=y)
    assert torch.equal(y, wc)
    wcg = model.causal_conv_grad(s["x"], s["w"], s["dy"])
    model.causal_conv_grad(a["x"], s["w"], a["dy"], dx=dx)
    assert torch.equal(dx, wcg.dx)
    z = torch.randn((1, 2, 5000), device="cuda").to(dtype)
    rows = room2.as_strided((1, 2, 5000), (2 * FAR, FAR, 1)).copy_(z)
    scores = torch.zeros((1, 2), device="cuda")
    assert same(model.beam_select(rows, scores, beams=9), model.beam_select(z, scores, beams=9))
    room.zero_()
    room[[0, -1]] = 3.0
    room[FAR] = 4.0
    norm, (out,) = model.clip_grad_norm([room], 17 ** 0.5)  # root of 34
    assert abs(float(norm) - 34 ** 0.5) < 1e-6 and out is room
    half = [float(v) for v in room[[0, FAR, -1]]]
    assert half == [float(torch.tensor(v * 0.5 ** 0.5).to(dtype)) for v in (3.0, 4.0, 3.0)]
    del room
    bits = room2[:1 << 31].view(2, 2, 1 << 29)
    bits[1, 1, -5:] = 7.0
    parents = torch.tensor([[1, 0], [0, 1]], dtype=torch.int32, device="cuda")
    (got,) = model.beam_reorder([bits], parents)
    assert torch.equal(got[1, 1, -9:], bits[1, 1, -9:]) and torch.equal(got[0, 0, :9], bits[0, 1, :9])
