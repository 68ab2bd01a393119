"""The sequence operators on the GPU against the oracle's 64-bit forms.

Tolerances are bounds on the rounding errors: each operation in fp32 is off by
at most U = 2^-24 relative to its result, an output by half a unit of its type
(u below) once more; sums of n terms are off by at most n U times the sum of
the terms' magnitudes, the gate's exponential and reciprocal by a few U.  The
oracle gives the magnitudes.
"""
import math

import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import seq as ref
from paper_2003_02989_amd import seq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": (torch.float32, 2.0 ** -24, 2.0 ** -149), "bf16": (torch.bfloat16, 2.0 ** -8, 2.0 ** -133),
         "f16": (torch.float16, 2.0 ** -11, 2.0 ** -24)}


def put(x, dtype):
    """(device tensor of dtype, the same values as float64 numpy)"""
    t = torch.as_tensor(np.ascontiguousarray(x)).to(dtype)
    return t.cuda(), t.double().numpy()


def check(name, got, want, tol):
    got = got.double().cpu().numpy().reshape(want.shape)
    assert np.all(np.isfinite(got)), f"{name}: not finite"
    err = np.abs(got - want)
    worst = float((err / np.maximum(tol, 1e-300)).max()) if err.size else 0.0
    say(f"{name}: error {float(err.max()) if err.size else 0:.3e}, {worst:.3f} of the tolerance")
    assert np.all(err <= tol), f"{name}: {worst:.2f} times the tolerance"


def rounded(want, extra, u, tiny):
    """Bound of an output's error: rounding to its type after an error `extra`."""
    return u * (np.abs(want) + extra) + extra + tiny


# ---------------------------------------------------------------- embedding

@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N,V,D,pad", [(1, 17, 64, 0), (16, 17, 64, 0), (37, 5, 1, 0), (130, 1025, 200, 3),
                                       (1000, 65, 331, 1), (9, 4, 2100, 0), (5, 1, 7, 0), (0, 3, 8, 0)])
def test_embed(ty, N, V, D, pad):
    dtype, u, tiny = TYPES[ty]
    rng = np.random.default_rng(N + V + D)
    t = rng.integers(-1, V + 1, N)  # -1: no shot; V: past the table
    table, tv = put(rng.standard_normal((V, D + pad)), dtype)
    out = seq.embed(torch.as_tensor(t).cuda(), table[:, :D], scale=1.3)
    want = ref.embed(t, tv[:, :D], float(np.float32(1.3)))
    check("embed", out, want, rounded(want, U * np.abs(want), u, tiny))
    assert torch.all(out[torch.as_tensor((t < 0) | (t >= V)).cuda()] == 0)


def shots(rng, kind, N, V):
    if kind == "uniform":
        return rng.integers(-1, V + 1, N)
    if kind == "two peaks":
        return np.where(rng.random(N) < 0.05, rng.integers(0, V, N), rng.integers(0, 2, N) * (V - 1))
    return np.full(N, V // 2) if kind == "one" else np.full(N, -1)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N,V,D,kind", [
    (1, 17, 64, "uniform"), (16, 1, 5, "uniform"), (64, 3, 8, "one"), (65, 3, 8, "one"), (129, 3, 33, "one"),
    (4096, 50, 16, "uniform"), (4097, 2047, 40, "uniform"), (5000, 2048, 7, "two peaks"), (9001, 65537, 12, "uniform"),
    (20000, 33, 331, "two peaks"), (300, 9, 600, "none"), (0, 5, 9, "none"), (140000, 6, 3, "two peaks")])
def test_embed_grad(ty, N, V, D, kind):
    dtype, u, tiny = TYPES[ty]
    rng = np.random.default_rng(N + V + D)
    t = shots(rng, kind, N, V)
    do, dv = put(0.1 * rng.standard_normal((N, D)), dtype)
    tok = torch.as_tensor(t).cuda()
    got = seq.embed_grad(tok, do, V, scale=0.7)
    again = seq.embed_grad(tok, do, V, scale=0.7)
    want, mag, n = ref.embed_grad(t, dv, V, float(np.float32(0.7)))
    # n additions, the piece sums' and the scale's rounding
    extra = (n[:, None] + 2) * U * mag
    check("embed_grad", got, want, rounded(want, extra, u, tiny))
    assert torch.equal(got, again)


def test_embed_grad_ignores_rows_without_a_token():
    do = torch.full((70, 9), float("nan"), device="cuda")
    do[3] = 1.0
    t = torch.full((70,), -1, dtype=torch.int64, device="cuda")
    t[3] = 2
    g = seq.embed_grad(t, do, 4)
    assert torch.equal(g, torch.tensor([0.0, 0, 1, 0], device="cuda")[:, None].expand(4, 9))
    e = seq.embed(t[:4], torch.full((3, 5), float("inf"), device="cuda"), scale=0.0)
    assert torch.all(e[:3] == 0)


def test_embed_of_a_table_past_32_bit_offsets():
    # 2^22 + 1 rows of 520 elements: the last rows lie past 2^31 elements
    V, D = (1 << 22) + 1, 520
    table = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    table[V - 1] = 3.0
    table[V - 2] = 2.0
    t = torch.tensor([V - 1, 0, V - 2], device="cuda")
    out = seq.embed(t, table)
    assert torch.equal(out[:, 0].float().cpu(), torch.tensor([3.0, 0, 2]))
    g = seq.embed_grad(t, out, V)
    assert torch.equal(g[V - 1], out[0]) and torch.equal(g[V - 2], out[2]) and float(g.abs().sum(dtype=torch.float32)) == 5 * D


# --------------------------------------------------------------- recurrence
# the error of a state obeys the recurrence itself, E_t = a E_{t-1} + k U M_t
# with M the magnitude of the state: at most k U T M in T steps, and as every
# a < 1 forgets, at most k U (1 / (1 - a)) M; K bounds both for the gates here
# (sigmoid of at most 6: 1 / (1 - a) <= 404) with k = 8 operations a step
K_SCAN = 8.0


def scan_factor(T):
    return K_SCAN * min(T + 8, 500) * U


def scan_inputs(rng, B, T, D, dtype, wide):
    both, bv = put(rng.standard_normal((B, T, 2 * D + wide)), dtype)
    g, gv = both[..., D:2 * D], np.clip(2 * bv[..., D:2 * D] + 1, -6, 6)
    g.copy_(torch.as_tensor(gv).to(dtype))
    return both[..., :D], g, bv[..., :D], g.double().cpu().numpy()


SCANS = [(1, 1, 64), (3, 1, 7), (2, 8, 130), (5, 9, 33), (2, 63, 64), (2, 64, 64), (3, 65, 129), (2, 200, 200),
         (1, 1000, 331), (1, 4099, 5), (70, 130, 20), (2, 2, 1)]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("B,T,D", SCANS)
def test_gated_scan_and_gradients(ty, ragged, B, T, D):
    dtype, u, tiny = TYPES[ty]
    rng = np.random.default_rng(B * T + D)
    x, g, xv, gv = scan_inputs(rng, B, T, D, dtype, 3)
    h0, h0v = put(rng.standard_normal((B, D)), torch.float32)
    n = None
    if ragged:
        n = rng.integers(0, T + 1, B)
        n[0] = 0 if B > 1 else T // 2
        n[-1] = T + 5 if B > 2 else n[-1]
        for b in range(B):  # what lies past the end is not looked at
            x[b, min(n[b], T):] = float("nan")
            g[b, min(n[b], T):] = float("inf")
    lengths = None if n is None else torch.as_tensor(n, dtype=torch.int32).cuda()
    y, h, states = seq.gated_scan(x, g, h0, lengths=lengths, keep=True)
    wy, wh, before, my, mh = ref.scan(xv, gv, h0v, n)
    k = scan_factor(T)
    check("y", y, wy, rounded(wy, k * my, u, tiny))
    check("h_last", h, wh, rounded(wh, k * mh, U, 0))
    ws = before[:, ::seq.SCAN_PIECE]
    kept = np.arange(ws.shape[1])[None] * seq.SCAN_PIECE < (np.full(B, T) if n is None else n)[:, None]
    states_kept = torch.where(torch.as_tensor(kept[..., None]).cuda(), states, torch.zeros((), device="cuda"))
    check("states", states_kept, ws * kept[..., None], rounded(ws, k * (np.abs(ws) + mh.max() + 4), U, 0))
    assert torch.equal(y, seq.gated_scan(x, g, h0, lengths=lengths)[0])
    # gradients
    dy, dyv = put(rng.standard_normal((B, T, D)), dtype)
    dh, dhv = put(rng.standard_normal((B, D)), torch.float32)
    if ragged:
        for b in range(B):
            dy[b, min(n[b], T):] = float("nan")
    dx, dg, dh0 = seq.gated_scan_grad(x, g, states, dy, dh_last=dh, lengths=lengths)
    wx, wg, w0, mx, mg, m0 = ref.scan_grad(xv, gv, h0v, n, dyv, dhv)
    check("dx", dx, wx, rounded(wx, k * mx, u, tiny))
    check("dg", dg, wg, rounded(wg, 2 * k * mg, u, tiny))
    check("dh0", dh0, w0, rounded(w0, k * m0, U, 0))


def test_gated_scan_without_optional_arguments():
    rng = np.random.default_rng(5)
    x, g, xv, gv = scan_inputs(rng, 2, 77, 40, torch.float32, 0)
    y, h, states = seq.gated_scan(x, g, keep=True)
    wy, wh, _, my, mh = ref.scan(xv, gv, None, None)
    check("y", y, wy, rounded(wy, scan_factor(77) * my, U, 0))
    dy, dyv = put(rng.standard_normal((2, 77, 40)), torch.float32)
    dx, dg, dh0 = seq.gated_scan_grad(x, g, states, dy)
    wx, wg, w0, mx, mg, m0 = ref.scan_grad(xv, gv, None, None, dyv, None)
    check("dx", dx, wx, rounded(wx, scan_factor(77) * mx, U, 0))
    check("dg", dg, wg, rounded(wg, 2 * scan_factor(77) * mg, U, 0))


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("T", [9, 16, 31])
def test_gated_scan_few_steps_of_many_channels(ty, T):
    test_gated_scan_and_gradients(ty, True, 1100, T, 480)


@pytest.mark.parametrize("ty", TYPES)
def test_gated_scan_step_by_step_in_place(ty):
    """Records extended step by step reach the states of one scan."""
    dtype, u, tiny = TYPES[ty]
    rng = np.random.default_rng(6)
    B, T, D = 5, 12, 75
    x, g, xv, gv = scan_inputs(rng, B, T, D, dtype, 1)
    n = rng.integers(0, T + 1, B)
    h = torch.zeros((B, D), device="cuda")
    ys = []
    for t in range(T):
        on = torch.as_tensor((t < n).astype(np.int32)).cuda()
        y, hh = seq.gated_scan(x[:, t:t + 1], g[:, t:t + 1], h, lengths=on, h_last=h)
        assert hh is h
        ys.append(y)
    wy, wh, _, my, mh = ref.scan(xv, gv, None, n)
    k = scan_factor(T)
    check("y", torch.cat(ys, 1), wy, rounded(wy, k * my, u, tiny))
    check("h", h, wh, rounded(wh, k * mh, U, 0))


@pytest.mark.parametrize("ty", TYPES)
def test_gated_scan_saturated_gates(ty):
    dtype = TYPES[ty][0]
    B, T, D = 1, 70, 66
    x = torch.arange(T, dtype=torch.float32, device="cuda")[None, :, None].expand(B, T, D).to(dtype).contiguous()
    g = torch.full((B, T, D), float("inf"), dtype=dtype, device="cuda")
    g[:, ::10] = float("-inf")  # take the input, then keep it for ten steps
    y, h, states = seq.gated_scan(x, g, keep=True)
    want = (torch.arange(T, device="cuda") // 10 * 10).float()[None, :, None].expand(B, T, D).to(dtype)
    assert torch.equal(y, want)
    dx, dg, dh0 = seq.gated_scan_grad(x, g, states, torch.ones_like(x))
    assert torch.equal(dx[0, :, 0].float().cpu(), torch.tensor([10.0 if t % 10 == 0 else 0.0 for t in range(T)]))
    assert torch.all(dg == 0) and torch.all(dh0 == 0)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("B,T,D", [(1, 20011, 331), (13, 3000, 200)])
def test_gated_scan_is_reproducible(ty, B, T, D):
    """The same bits whatever the order in which segments finish."""
    dtype = TYPES[ty][0]
    x, g = torch.randn((2, B, T, D), device="cuda").to(dtype).unbind(0)
    g = (g * 2 + 3).to(dtype)
    dy, dh = torch.randn((B, T, D), device="cuda").to(dtype), torch.randn((B, D), device="cuda")
    want = None
    for _ in range(6):
        y, h, states = seq.gated_scan(x, g, keep=True)
        out = (y, h, states) + seq.gated_scan_grad(x, g, states, dy, dh_last=dh)
        want = want or [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_gated_scan_nothing_to_do():
    z = torch.zeros((2, 0, 5), device="cuda")
    h0 = torch.ones((2, 5), device="cuda")
    y, h, states = seq.gated_scan(z, z, h0, keep=True)
    assert y.shape == (2, 0, 5) and torch.equal(h, h0) and states.shape == (2, 0, 5)
    assert torch.equal(seq.gated_scan_grad(z, z, states, z, dh_last=h0)[2], h0)
    e = torch.zeros((0, 4, 5), device="cuda")
    assert seq.gated_scan(e, e)[0].shape == (0, 4, 5)


# --------------------------------------------------------------- layer norm
# sums in fp32: at most 40 additions in a row (32 in a lane, 6 across lanes),
# so mean and variance are off by at most 40 U of their magnitudes; values far
# from zero lose rms(x) / sigma of that
@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("N,D,pad", [(1, 1, 0), (1, 64, 0), (64, 200, 0), (33, 331, 5), (7, 512, 0), (513, 40, 0),
                                     (5, 1000, 8), (3, 1024, 0), (9, 2047, 1), (2, 4096, 0), (3, 8200, 0),
                                     (2, 17001, 0), (0, 8, 0), (1500, 16, 0)])
def test_layer_norm_and_gradients(ty, bias, N, D, pad):
    dtype, u, tiny = TYPES[ty]
    rng = np.random.default_rng(N + D)
    eps = 1e-5
    x, xv = put(rng.standard_normal((N, D + pad)) * 1.5 + 0.3, dtype)
    x, xv = x[:, :D], xv[:, :D]
    w, wv = put(1 + 0.2 * rng.standard_normal(D), dtype)
    b, bv = put(0.2 * rng.standard_normal(D), dtype)
    y, mean, rstd = seq.layer_norm(x, w, b if bias else None, eps=eps, keep=True)
    e32 = float(np.float32(eps))
    if N:
        wy, wm, wr = ref.norm(xv, wv, bv if bias else None, e32)
    else:
        wy, wm, wr = np.zeros((0, D)), np.zeros(0), np.zeros(0)
    rms = np.sqrt((xv ** 2).mean(1)) if N else np.zeros(0)
    loss = (1 + rms * wr)[:, None]  # digits lost to the mean
    xh = (xv - wm[:, None]) * wr[:, None]
    k = 64 * U
    ey = k * loss * np.abs(wv) * (1 + np.abs(xh)) * loss + k * (np.abs(bv) if bias else 0)
    check("y", y, wy, rounded(wy, ey, u, tiny))
    check("mean", mean, wm, k * rms + 1e-30)
    check("rstd", rstd, wr, k * wr * loss[:, 0] ** 2)
    assert torch.equal(y, seq.layer_norm(x, w, b if bias else None, eps=eps))
    dy, dv = put(rng.standard_normal((N, D)), dtype)
    dx, dw, db = seq.layer_norm_grad(x, w, mean, rstd, dy)
    wx, ww, wb = ref.norm_grad(xv, wv, e32, dv) if N else (np.zeros((0, D)), np.zeros(D), np.zeros(D))
    uu = np.abs(dv * wv)
    m1 = uu.mean(1)[:, None] if N else np.zeros((0, 1))
    m2 = (uu * (np.abs(xh) + 1)).mean(1)[:, None] if N else np.zeros((0, 1))
    ex = 4 * k * loss ** 2 * wr[:, None] * (uu + m1 + (np.abs(xh) + 1) * m2)
    check("dx", dx, wx, rounded(wx, ex, u, tiny))
    ew = ((k * loss ** 2 + N * U) * np.abs(dv) * (np.abs(xh) + 1)).sum(0)
    check("dweight", dw, ww, rounded(ww, ew, u, tiny))
    check("dbias", db, wb, rounded(wb, (N + 16) * U * np.abs(dv).sum(0), u, tiny))


def test_layer_norm_keeps_bad_rows_to_themselves():
    x = torch.randn((6, 100), device="cuda")
    x[2, 5] = float("nan")
    x[4, 7] = float("inf")
    w = torch.ones(100, device="cuda")
    y = seq.layer_norm(x, w)
    good = [0, 1, 3, 5]
    assert torch.isfinite(y[good]).all() and not torch.isfinite(y[2]).any()
    assert torch.equal(y[good], seq.layer_norm(x[good].contiguous(), w))


# ------------------------------------------------------------ cross entropy

XENTS = [(1, 17, 64), (4, 65, 200), (16, 129, 33), (17, 40, 7), (40, 1000, 130), (64, 257, 1), (65, 300, 64),
         (130, 129, 200), (300, 1025, 128), (257, 2000, 331), (700, 33, 65), (3, 1, 5), (100, 5000, 256)]


def xent_inputs(rng, N, V, D, dtype):
    h, hv = put(rng.standard_normal((N, D + 3)), dtype)
    W, Wv = put(2 / math.sqrt(D) * rng.standard_normal((V, D + 1)), dtype)
    t = rng.integers(-1, V + 1, N)
    t[rng.random(N) < 0.2] = -1
    return h[:, :D], hv[:, :D], W[:, :D], Wv[:, :D], t


def logit_error(ty, hv, Wv):
    """fp32 sums of D products; fp32 inputs hold 22 bits each (2^-22 a side, and
    2^-22 for the left-out product)."""
    m = np.abs(hv) @ np.abs(Wv).T
    D = hv.shape[1]
    return (D * U + (3 * 2.0 ** -22 if ty == "f32" else 0)) * m


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N,V,D", XENTS)
def test_softmax_xent_and_gradients(ty, N, V, D):
    dtype, u, tiny = TYPES[ty]
    rng = np.random.default_rng(N + V + D)
    h, hv, W, Wv, t = xent_inputs(rng, N, V, D, dtype)
    tok = torch.as_tensor(t).cuda()
    loss, lse = seq.softmax_xent(h, W, tok)
    wl, ws, z = ref.xent(hv, Wv, t)
    ez = logit_error(ty, hv, Wv)
    # sums of V exponentials of arguments down to -max|z|, a logarithm
    es = ez.max(1) + (V + 32) * U + 4 * U * np.abs(z).max(1)
    check("lse", lse, ws, es)
    ok = (t >= 0) & (t < V)
    check("loss", loss, wl, np.where(ok, 2 * es, 0))
    up, upv = put(rng.standard_normal(N) / N, torch.float32)
    dh, dW, gl, gs = seq.softmax_xent_grad(h, W, tok, up)
    wdh, wdW, _, _, p = ref.xent_grad(hv, Wv, t, upv)
    check("lse with gradients", gs, ws, es)
    check("loss with gradients", gl, wl, np.where(ok, 2 * es, 0))
    # an entry of p: the logit's and lse's errors and its exponential's times
    # exp(z - lse), its rounding to 16 bits (in two parts for fp32: 2^-22)
    up16 = 2.0 ** -21 if ty == "f32" else u
    pe = np.abs(upv)[:, None] * np.exp(z - ws[:, None]) * (ez + es[:, None] + 16 * U * (1 + np.abs(z - ws[:, None])))
    pe = pe + 2 * up16 * np.abs(p) + 2.0 ** -38 * np.abs(upv).max()
    pe[~ok] = 0
    w22 = 3 * 2.0 ** -22 if ty == "f32" else 0
    eh = pe @ np.abs(Wv) + ((V + 64) * U + w22) * (np.abs(p) @ np.abs(Wv))
    check("dhidden", dh, wdh, rounded(wdh, eh, u, tiny))
    hz = np.where(ok[:, None], np.abs(hv), 0)
    ew = pe.T @ hz + ((N + 64) * U + w22) * (np.abs(p).T @ hz)
    check("dweight", dW, wdW, rounded(wdW, ew, u, tiny))
    assert torch.all(dh[torch.as_tensor(~ok).cuda()] == 0)
    again = seq.softmax_xent_grad(h, W, tok, up)
    assert torch.equal(dh, again[0]) and torch.equal(dW, again[1])


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N,V,D", [(4200, 4100, 40), (4099, 1025, 300), (2500, 4097, 33), (600, 9001, 260)])
def test_softmax_xent_many_tiles(ty, N, V, D):
    """More tiles than compute units, and last rounds cut in two, in four and not at all."""
    test_softmax_xent_and_gradients(ty, N, V, D)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N", [16, 17, 33])
def test_softmax_xent_few_tokens_of_whole_pieces(ty, N):
    test_softmax_xent_and_gradients(ty, N, 300, 128)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N", [5, 200])
def test_softmax_xent_bad_rows_without_targets(ty, N):
    """Rows without a target may hold anything; so may their upstream."""
    dtype = TYPES[ty][0]
    rng = np.random.default_rng(8)
    V, D = 150, 64
    h, hv, W, Wv, t = xent_inputs(rng, N, V, D, dtype)
    t[0], t[1] = 3, -1
    bad = torch.as_tensor((t < 0) | (t >= V)).cuda()
    tok, up = torch.as_tensor(t).cuda(), torch.rand(N, device="cuda")
    clean = seq.softmax_xent_grad(h, W, tok, up)
    h2, up2 = h.clone(), up.clone()
    h2[bad] = float("nan")
    up2[bad] = float("inf")
    dh, dW, loss, lse = seq.softmax_xent_grad(h2, W, tok, up2)
    assert torch.equal(dW, clean[1]) and torch.equal(dh[~bad], clean[0][~bad]) and torch.all(dh[bad] == 0)
    assert torch.equal(loss, clean[2]) and torch.all(loss[bad] == 0)
    # no target at all
    none = torch.full_like(tok, -1)
    dh, dW, loss, _ = seq.softmax_xent_grad(h2, W, none, up2)
    assert torch.all(dh == 0) and torch.all(dW == 0) and torch.all(loss == 0)


@pytest.mark.parametrize("ty", TYPES)
def test_softmax_xent_confident_rows(ty):
    """Logits of hundreds, one far above the others: finite, and p - 1 of a
    probability near one is small, not rounded away."""
    dtype = TYPES[ty][0]
    V, D, N = 300, 64, 96
    W = torch.zeros((V, D), dtype=dtype, device="cuda")
    W[:D] = 16 * torch.eye(D, dtype=dtype, device="cuda")
    h = (16 * torch.eye(D, dtype=dtype, device="cuda")).repeat(2, 1)[:N].contiguous()
    t = torch.arange(N, device="cuda") % D
    loss, lse = seq.softmax_xent(h, W, t)
    assert torch.all(lse == 256) and torch.all(loss == 0)
    dh, dW, loss, lse = seq.softmax_xent_grad(h, W, t, torch.ones(N, device="cuda"))
    assert torch.all(dh == 0) and torch.all(dW == 0) and torch.all(loss == 0)
    wrong = (t + 1) % D
    loss = seq.softmax_xent(h, W, wrong)[0]
    assert torch.all(loss == 256)


def test_softmax_xent_fp32_rows_of_any_magnitude():
    """fp32 inputs whose rows and columns differ by many powers of ten."""
    rng = np.random.default_rng(9)
    N, V, D = 150, 140, 96
    hv = rng.standard_normal((N, D)) * 10.0 ** rng.integers(-20, 1, (N, 1))
    Wv = rng.standard_normal((V, D)) * 10.0 ** rng.integers(-18, 1, (V, 1))
    h, hv = put(hv, torch.float32)
    W, Wv = put(Wv, torch.float32)
    t = rng.integers(0, V, N)
    loss, lse = seq.softmax_xent(h, W, torch.as_tensor(t).cuda())
    wl, ws, z = ref.xent(hv, Wv, t)
    es = logit_error("f32", hv, Wv).max(1) + (V + 32) * U + 4 * U * np.abs(z).max(1)
    check("lse", lse, ws, es)
    up = np.full(N, 1.0 / N)
    dh, dW, _, _ = seq.softmax_xent_grad(h, W, torch.as_tensor(t).cuda(), put(up, torch.float32)[0])
    wdh, wdW, _, _, p = ref.xent_grad(hv, Wv, t, np.float32(up).astype(float))
    # relative to the largest of a column: what the other operand's scale resolves
    check("dhidden", dh, wdh, 1e-5 * np.abs(wdh).max() + 0 * wdh)
    check("dweight", dW, wdW, 1e-5 * np.abs(wdW).max() + 0 * wdW)


def test_softmax_xent_without_tokens():
    W = torch.ones((7, 5), device="cuda")
    e = torch.zeros((0, 5), device="cuda")
    t = torch.zeros((0,), dtype=torch.int64, device="cuda")
    dh, dW, loss, lse = seq.softmax_xent_grad(e, W, t, torch.zeros(0, device="cuda"))
    assert dh.shape == (0, 5) and torch.all(dW == 0) and loss.numel() == 0
    assert seq.softmax_xent(e, W, t)[0].numel() == 0


# ------------------------------------------------------------------- streams

def test_other_streams_and_graphs():
    """Calls on a stream of their own, and captured calls replayed on new data."""
    rng = np.random.default_rng(10)
    B, T, D, V = 3, 150, 40, 70
    tok = torch.as_tensor(rng.integers(-1, V, (B, T))).cuda()
    table = torch.randn((V, 2 * D), device="cuda")
    W = torch.randn((V, D), device="cuda")
    w = torch.ones(D, device="cuda")
    up = torch.full((B, T), 1.0 / (B * T), device="cuda")
    nxt = torch.roll(tok, -1, 1).contiguous()

    def step(stream=None):
        e = seq.embed(tok, table, scale=0.5, stream=stream)
        y, _, states = seq.gated_scan(e[..., :D], e[..., D:], keep=True, stream=stream)
        o, mean, rstd = seq.layer_norm(y, w, keep=True, stream=stream)
        dh, dW, loss, _ = seq.softmax_xent_grad(o, W, nxt, up, stream=stream)
        dy, dw, db = seq.layer_norm_grad(y, w, mean, rstd, dh, stream=stream)
        de = torch.empty_like(e)
        seq.gated_scan_grad(e[..., :D], e[..., D:], states, dy, dx=de[..., :D], dg=de[..., D:], stream=stream)
        return loss, dW, dw, seq.embed_grad(tok, de, V, scale=0.5, stream=stream)

    want = [o.clone() for o in step()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = step(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        table.copy_(torch.randn((V, 2 * D), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), k
