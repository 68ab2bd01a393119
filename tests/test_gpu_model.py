"""The operators of selective models on the GPU against the oracle's 64-bit forms.

Tolerances are bounds on the rounding errors: an operation in fp32 is off by at
most U = 2^-24 relative to its result, an output by half a unit of its type (u)
once more; sums of n terms by at most n U times the sum of the terms' magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import model as ref
from paper_2003_02989_amd import model
from test_gpu_seq import TYPES, U, check, put, rounded

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------- selective scan

class Scan:
    """Inputs of a selective scan on the device and in float64: strided views,
    what lies past the records' lengths NaN."""

    def __init__(self, ty, B, T, D, S, ragged=True, gated=True, seed=0):
        self.dtype, self.u, self.tiny = TYPES[ty]
        rng = np.random.default_rng(B + T + D + S + seed)
        self.n = rng.integers(0, T + 1, B) if ragged else None
        if ragged and B > 2:
            self.n[0], self.n[1] = 0, T
        parts = rng.standard_normal((B, T, 3 * D + 2 * S + 1))
        if ragged:
            parts[np.arange(T) >= self.n[:, None]] = np.nan
        p, pv = put(parts, self.dtype)
        cut = np.cumsum([0, D, D, D, S, S])
        (self.x, self.dt, self.z, self.B, self.C) = (p[..., a:b] for a, b in zip(cut, cut[1:]))
        (self.xv, self.dtv, self.zv, self.Bv, self.Cv) = (pv[..., a:b] for a, b in zip(cut, cut[1:]))
        f = torch.float32
        self.A, self.Av = put(-np.exp(rng.standard_normal((D, S))), f)
        self.skip, self.skipv = put(rng.standard_normal(D), f)
        self.bias, self.biasv = put(rng.uniform(-4, 0, D), f)
        self.h0, self.h0v = put(rng.standard_normal((B, D, S)), f)
        self.dh, self.dhv = put(rng.standard_normal((B, D, S)), f)
        dy = rng.standard_normal((B, T, D))
        if ragged:
            dy[np.arange(T) >= self.n[:, None]] = np.nan
        self.dy, self.dyv = put(dy, self.dtype)
        if not gated:
            self.z = self.zv = self.skip = self.skipv = self.bias = self.biasv = None
        self.lengths = None if self.n is None else torch.as_tensor(self.n.astype(np.int32)).cuda()
        self.args = (self.x, self.dt, self.A, self.B, self.C)
        self.more = dict(skip=self.skip, z=self.z, dt_bias=self.bias, lengths=self.lengths)
        self.values = (self.xv, self.dtv, self.Av, self.Bv, self.Cv, self.skipv, self.zv, self.biasv)

    def forward(self, h0=True, **kw):
        return model.selective_scan(*self.args, h0=self.h0 if h0 else None, **self.more, **kw)

    def check_forward(self, y, h, h0=True):
        wy, wh, wp, _, (pm, pe, m, e) = ref.selective_scan(*self.values, self.h0v if h0 else None, self.n)
        # z sigmoid(z): 6 units; errors of second order: doubled
        gate = 1 if self.zv is None else np.abs(np.nan_to_num(self.zv * ref.sigmoid(self.zv)))
        check("y", y, wy, rounded(wy, 2 * U * gate * (pe + 6 * pm), self.u, self.tiny))
        check("h_last", h, wh, 2 * U * e[:, -1] + U * np.abs(wh) + 2.0 ** -126)

    def grads(self, states, dh=True):
        return model.selective_scan_grad(*self.args, states, self.dy, dh_last=self.dh if dh else None, **self.more)

    def check_grads(self, g, dh=True, h0=True):
        a = (*self.values, self.h0v if h0 else None, self.n, self.dyv, self.dhv if dh else None)
        want, size = ref.selective_scan_grad(*a), ref.selective_scan_grad(*a, absolute=True)
        B, T, D = self.xv.shape
        S = self.Av.shape[1]
        # every term is a product along a path of at most T steps, forwards and then
        # backwards: 3 units a step and its decays' exponents' errors, 24 + |v| units
        # of their sum (whose exponential leaves nothing past 30); the path's ends
        # are a few more, sums over states, channels and steps one a term
        on = np.ones((B, T)) if self.n is None else np.arange(T) < self.n[:, None]
        v = np.where(on[..., None], self.dtv + (0 if self.biasv is None else self.biasv), -np.inf)
        reach = (ref.softplus(v).sum(1)[..., None] * np.abs(self.Av)).max() if B * T else 0
        off = 24 + np.abs(np.where(np.isfinite(v), v, 0)).max(initial=0)
        k = 2 * U * (2 * 4 * T + off * min(reach, 30) + 2 * off + 20 + S)
        terms = {"dB": D, "dC": D, "dA": B * T, "dskip": B * T, "ddt_bias": B * T}
        for name, w, m in zip(("dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "ddt_bias", "dh0"), want, size):
            got = getattr(g, name)
            if got is None:
                assert name in ("dz", "dskip", "ddt_bias") and self.zv is None
                continue
            f32 = name in ("dA", "dskip", "ddt_bias", "dh0")
            u, tiny = (U, 2.0 ** -126) if f32 else (self.u, max(self.tiny, 2.0 ** -126))
            check(name, got, w, rounded(w, (k + terms.get(name, 0) * U) * m, u, tiny))


SCANS = [(1, 1, 5, 1), (3, 1, 70, 16), (2, 7, 64, 4), (4, 16, 65, 16), (3, 17, 130, 5), (3, 40, 33, 64), (4, 33, 70, 33),
         (2, 50, 10, 20), (1, 300, 20, 16), (2, 1000, 9, 3), (5, 450, 66, 9), (3, 0, 7, 4), (70, 2, 3, 2)]


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("B,T,D,S", SCANS)
def test_selective_scan_and_gradients(ty, B, T, D, S):
    c = Scan(ty, B, T, D, S)
    y, h, states = c.forward(keep=True)
    c.check_forward(y, h)
    y2, h2 = c.forward()
    assert torch.equal(y, y2) and torch.equal(h, h2)
    c.check_grads(c.grads(states))


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("B,T,D,S", [(2, 37, 70, 16), (1, 400, 12, 6), (3, 1, 9, 16)])
def test_selective_scan_without_the_optional_inputs(ty, B, T, D, S):
    c = Scan(ty, B, T, D, S, ragged=False, gated=False, seed=1)
    y, h, states = c.forward(h0=False, keep=True)
    c.check_forward(y, h, h0=False)
    c.check_forward(*c.forward(h0=False), h0=False)
    c.check_grads(c.grads(states, dh=False), dh=False, h0=False)
