"""The operators of selective models at sizes where their kernels' loops are taken
more than once: long runs of a convolution, threads and workgroups with several
runs or records, chunks of time with many states, several records a thread.

Most inputs are whole numbers (the scan's steps are 32 exactly, its decays one or
nothing), so that every sum is formed without rounding, whatever its order, and
outputs have to be the formula's to the last bit.  The formulas are written out here
in 64 bits over whole arrays.
"""
import numpy as np
import pytest
import torch

from paper_2003_02989_amd import model
from test_gpu_model import Scan
from test_gpu_seq import TYPES, U

pytestmark = pytest.mark.gpu


def whole(gen, shape, most, density=1.0):
    """Whole numbers from -most to most, zeros but for a part."""
    v = torch.randint(-most, most + 1, shape, generator=gen, device="cuda").double()
    return v if density == 1.0 else v * (torch.rand(shape, generator=gen, device="cuda") < density)


def same(name, got, want):
    assert got.shape == want.shape, name
    wrong = got != want.to(got.dtype)
    assert not wrong.any(), f"{name}: {int(wrong.sum())} of {wrong.numel()} differ, first at {wrong.nonzero()[0].tolist()}"


def near(name, got, want, tol):
    worst = float(((got.double() - want).abs() / tol).max())
    assert worst <= 1, f"{name}: {worst:.2f} times the tolerance"  # NaN is not


# --------------------------------------------------------- causal convolution

# B, T, D, taps; steps of a run: forward, gradient
CONVS = [(2100, 1000, 9, 4, 16, 64), (2100, 1000, 9, 6, 16, 64), (2100, 1000, 9, 8, 16, 64), (8200, 1030, 9, 2, 64, 64),
         (8200, 1030, 9, 7, 64, 64), (2100, 700, 3, 5, 16, 16), (4200, 1000, 1, 8, 16, 32)]


class Conv:
    """Inputs on the device, NaN past the lengths, and the same in 64 bits, zeros there."""

    def __init__(self, ty, B, T, D, K, ragged, values):
        dtype = TYPES[ty][0]
        gen = torch.Generator(device="cuda")
        gen.manual_seed(B + T + D + K)
        self.n = torch.full((B,), T, device="cuda")
        if ragged:
            self.n = torch.randint(0, T + 1, (B,), generator=gen, device="cuda")
            self.n[:4] = torch.tensor([0, T, 1, T - 1])
        past = torch.arange(T, device="cuda")[None, :, None] >= self.n[:, None, None]

        def make(shape, most):
            v = whole(gen, shape, most) if values == "whole" else torch.randn(shape, generator=gen, device="cuda").double()
            v = v.to(dtype)
            return v, v.double()
        x, self.xv = make((B, T, D), 1)
        dy, self.dyv = make((B, T, D), 1)
        self.x, self.dy = x.masked_fill(past, float("nan")), dy.masked_fill(past, float("nan"))
        self.xv.masked_fill_(past, 0)
        self.dyv.masked_fill_(past, 0)
        (self.w, self.wv), (self.bias, self.biasv) = make((K, D), 2), make((D,), 2)
        (self.state, self.statev), (self.dlast, self.dlastv) = make((B, K - 1, D), 1), make((B, K - 1, D), 2)
        self.on = ~past
        self.more = dict(bias=self.bias, state=self.state, lengths=self.n.int() if ragged else None)

    def ends(self):
        """Places of the K - 1 inputs before the step after each record's last."""
        K = self.w.shape[0]
        at = self.n[:, None] + torch.arange(K - 1, device="cuda")
        return at[:, :, None].expand(-1, -1, self.x.shape[2])

    def forward(self):
        """u, the sum of its terms' magnitudes, the inputs with the state before them"""
        T = self.x.shape[1]
        xs = torch.cat((self.statev, self.xv), 1)
        u, um = self.biasv + torch.zeros_like(self.xv), self.biasv.abs() + torch.zeros_like(self.xv)
        for k, w in enumerate(self.wv):
            term = w * xs[:, k:k + T]
            u += term
            um += term.abs()
        return u, um, xs

    def backward(self, g, xs, absolute=False):
        """dx, dweight, dbias, dstate of u's gradient g"""
        f = torch.abs if absolute else lambda v: v
        K, T = self.wv.shape[0], self.x.shape[1]
        back = torch.zeros_like(xs)
        back.scatter_add_(1, self.ends(), f(self.dlastv))
        for k, w in enumerate(self.wv):
            back[:, k:k + T] += f(w) * g
        dw = torch.stack([(g * f(xs[:, k:k + T])).sum((0, 1)) for k in range(K)])
        return back[:, K - 1:] * self.on, dw, g.sum((0, 1)), back[:, :K - 1]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,T,D,K", [c[:4] for c in CONVS])
def test_causal_conv_of_whole_numbers(ty, B, T, D, K, ragged):
    c = Conv(ty, B, T, D, K, ragged, "whole")
    u, _, xs = c.forward()
    y, last = model.causal_conv(c.x, c.w, silu=False, **c.more)
    same("y", y, u * c.on)
    same("last", last, xs.gather(1, c.ends()))
    g = model.causal_conv_grad(c.x, c.w, c.dy, dlast=c.dlast, silu=False, **c.more)
    for name, w in zip(("dx", "dweight", "dbias", "dstate"), c.backward(c.dyv, xs)):
        same(name, getattr(g, name), w)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,T,D,K", [c[:4] for c in CONVS])
def test_causal_conv_with_silu_in_long_runs(ty, B, T, D, K, ragged):
    """The bounds of test_gpu_model.py, but for the sums over all steps: a thread adds
    up two runs of 64 at most, 64 groups every 64th of 2^19 / 5 threads or fewer (for
    one channel 2^19), seven levels their sums."""
    c = Conv(ty, B, T, D, K, ragged, "normal")
    _, r, tiny = TYPES[ty]
    u, um, xs = c.forward()
    s = torch.sigmoid(u)
    want = u * s * c.on
    y, _ = model.causal_conv(c.x, c.w, **c.more)
    extra = 1.1 * (K + 1) * U * um + (8 + u.abs()) * U * want.abs()
    near("y", y, want, r * (want.abs() + extra) + extra + tiny)
    most = float((u * c.on).abs().max())
    g = model.causal_conv_grad(c.x, c.w, c.dy, dlast=c.dlast, **c.more)
    wants = c.backward(c.dyv * (s + u * s * (1 - s)), xs)
    sizes = c.backward(c.dyv.abs() * (s + u.abs() * s * (1 - s) + um), xs, absolute=True)
    depth = 128 + (2 ** 19 // max(1, (D + 1) // 2) + 63) // 64 + 7
    for name, w, m in zip(("dx", "dweight", "dbias", "dstate"), wants, sizes):
        extra = (2 * K + 14 + 2 * most + (depth if name in ("dweight", "dbias") else 0)) * U * m
        near(name, getattr(g, name), w, r * (w.abs() + extra) + extra + tiny)


# ------------------------------------------------------------- selective scan

# B, T, D, S, chunks of time, with lengths; what is worked on twice
EXACT = [(4200, 3, 5, 3, 1, True), (4200, 20, 5, 3, 1, True), (150, 5, 2048, 17, 1, True), (2100, 9, 70, 40, 1, True),
         (150, 4, 2048, 17, 1, False), (8, 6600, 300, 4, 104, True), (3, 656, 5, 3, 41, True), (3, 656, 5, 3, 41, False),
         (2, 500, 40, 20, 16, True), (1, 700, 70, 33, 22, True), (3, 450, 9, 64, 15, True), (2, 1312, 9, 64, 82, False)]


def exact_set(dtype, B, T, D, S, ragged):
    """(the call's arguments, the same in 64 bits): steps of 32, d x_t whole, channels'
    states that either stay (A = 0) or are gone after a step (exp(-256) is nothing in
    fp32)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(B + T + D + S)
    n = torch.full((B,), T, device="cuda")
    if ragged:
        n = torch.randint(0, T + 1, (B,), generator=gen, device="cuda")
        n[torch.arange(min(B, 3))] = torch.tensor([T, 0, T // 2], device="cuda")[:min(B, 3)]
    past = (torch.arange(T, device="cuda") >= n[:, None])[..., None]
    sparse = min(1.0, 40 / max(T, 1))
    v = {"x": whole(gen, (B, T, D), 1, sparse) / 32, "B": whole(gen, (B, T, S), 1), "C": whole(gen, (B, T, S), 1),
         "dy": whole(gen, (B, T, D), 1, sparse), "skip": 32 * whole(gen, (D,), 1), "dt_bias": whole(gen, (D,), 4),
         "A": -8.0 * torch.randint(0, 2, (D, S), generator=gen, device="cuda").double(),
         "h0": whole(gen, (B, D, S), 1), "dh": whole(gen, (B, D, S), 1), "n": n}
    v["dt"] = (32 - v["dt_bias"]).expand(B, T, D)
    nan = float("nan")
    t = {k: v[k].masked_fill(past, nan).to(dtype) for k in ("x", "dt", "B", "C", "dy")}
    t.update({k: v[k].float() for k in ("A", "skip", "dt_bias", "h0", "dh")})
    t["lengths"] = n.int() if ragged else None
    return t, v


def exact_scan(v):
    """The formulas step by step, in 64 bits, over all records, channels and states; of
    every sum that the kernels form the magnitudes' sum as well."""
    B, T, D = v["x"].shape
    keep = (v["A"] == 0).double()
    on = (torch.arange(T, device="cuda") < v["n"][:, None]).double()
    h = torch.empty((T + 1,) + v["h0"].shape, dtype=torch.float64, device="cuda")
    h[0] = v["h0"]
    y = torch.zeros_like(v["x"])
    for t in range(T):
        go = on[:, t, None, None]
        new = keep * h[t] + (32 * v["x"][:, t])[..., None] * v["B"][:, t, None]
        h[t + 1] = go * new + (1 - go) * h[t]
        y[:, t] = on[:, t, None] * ((h[t + 1] * v["C"][:, t, None]).sum(-1) + v["skip"] * v["x"][:, t])
    g = {k: torch.zeros_like(v[s]) for k, s in (("dx", "x"), ("ddt", "x"), ("dB", "B"), ("dC", "C"), ("dA", "A"))}
    size = torch.zeros_like(v["A"])
    m = v["dh"].clone()
    for t in range(T - 1, -1, -1):
        go = on[:, t, None, None]
        q, x = on[:, t, None] * v["dy"][:, t], v["x"][:, t]
        l = go * (v["C"][:, t, None] * q[..., None] + m)
        bl = (v["B"][:, t, None] * l).sum(-1)
        g["dC"][:, t] = (q[..., None] * h[t + 1]).sum(1)
        g["dB"][:, t] = ((32 * x)[..., None] * l).sum(1)
        g["dx"][:, t] = on[:, t, None] * (32 * bl + v["skip"] * q)
        g["ddt"][:, t] = on[:, t, None] * x * bl
        w = keep * l * h[t]
        g["dA"] += 32 * w.sum(0)
        size += w.abs().sum(0)
        m = go * keep * l + (1 - go) * m
    g["dskip"] = (on[..., None] * v["dy"] * v["x"]).sum((0, 1))
    g["ddt_bias"] = g["ddt"].sum((0, 1))
    g["dh0"] = m
    assert float(size.max()) < 2 ** 24 and float(h.abs().max()) * v["A"].shape[1] < 2 ** 24  # sums without rounding
    return y, h, g


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("B,T,D,S,ragged", [c[:4] + c[5:] for c in EXACT])
def test_selective_scan_of_whole_numbers(ty, B, T, D, S, ragged):
    t, v = exact_set(TYPES[ty][0], B, T, D, S, ragged)
    wy, wh, wg = exact_scan(v)
    args = (t["x"], t["dt"], t["A"], t["B"], t["C"])
    more = dict(skip=t["skip"], dt_bias=t["dt_bias"], lengths=t["lengths"])
    y, h, states = model.selective_scan(*args, h0=t["h0"], keep=True, **more)
    same("y", y, wy)
    same("h_last", h, wh[T])
    pieces = -(-T // 16)
    begun = (16 * torch.arange(pieces, device="cuda") < v["n"][:, None])[..., None, None]  # the others are not written
    want = wh[:T:16].permute(1, 0, 3, 2)
    same("states", torch.where(begun, states, 0), torch.where(begun, want, 0))
    g = model.selective_scan_grad(*args, states, t["dy"], dh_last=t["dh"], **more)
    for name in ("dx", "dA", "dB", "dC", "dskip", "dh0"):
        same(name, getattr(g, name), wg[name])
    # these have a factor sigmoid(32), a reciprocal of one off by a unit at most
    size = wg["ddt"].abs()
    near("ddt", g.ddt, wg["ddt"], TYPES[ty][1] * size + 4 * U * size + 2.0 ** -149)
    near("ddt_bias", g.ddt_bias, wg["ddt_bias"], 1000 * U * size.sum((0, 1)) + 2.0 ** -149)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("B,T,D,S", [(2, 500, 40, 20), (1, 450, 70, 33), (3, 420, 9, 64), (3, 656, 5, 3)])
def test_selective_scan_of_many_states_in_chunks(ty, B, T, D, S):
    """Decays and gates of all sizes, against the oracle."""
    c = Scan(ty, B, T, D, S, seed=2)
    y, h, states = c.forward(keep=True)
    c.check_forward(y, h)
    c.check_grads(c.grads(states))


# B, D, S: in fp32 with more than four states a thread takes four records
STEPS = [(4097, 512, 3), (2049, 512, 5), (1027, 512, 16), (513, 512, 20), (259, 512, 64), (2731, 600, 4)]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("B,D,S", STEPS)
@pytest.mark.parametrize("ragged", [False, True])
def test_single_steps_of_many_records(ty, B, D, S, ragged):
    c = Scan(ty, B, 1, D, S, ragged=ragged, seed=3)
    y, h = c.forward()
    c.check_forward(y, h)
    y2, h2, _ = c.forward(keep=True)  # by the tiled form, which gives the same bits
    assert torch.equal(y, y2) and torch.equal(h, h2)
    if ragged:
        stays = c.lengths == 0
        assert torch.equal(h[stays], c.h0[stays]) and not y[stays].any() and int(stays.sum()) > 0
    kept = c.h0.clone()
    y2, _ = model.selective_scan(*c.args, h0=kept, h_last=kept, **c.more)
    assert torch.equal(y, y2) and torch.equal(h, kept)
    assert np.isfinite(float(h.sum()))
