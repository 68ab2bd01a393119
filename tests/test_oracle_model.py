"""The 64-bit operators of selective models of the oracle: gradients against
central differences, and closed forms."""
import numpy as np
import pytest

from oracle import model as ref
from test_oracle_seq import TOL, differences


@pytest.mark.parametrize("lengths", [None, [5, 0, 2]])
@pytest.mark.parametrize("gated", [True, False])
def test_selective_scan_gradients_match_differences(lengths, gated):
    rng = np.random.default_rng(7)
    B, T, D, S = 3, 5, 2, 3
    x, dt, z, dy = (rng.standard_normal((B, T, D)) for _ in range(4))
    Bm, Cm = rng.standard_normal((2, B, T, S))
    A = -np.exp(rng.standard_normal((D, S)))
    skip, bias = rng.standard_normal((2, D))
    h0, dh = rng.standard_normal((2, B, D, S))
    n = None if lengths is None else np.array(lengths)
    if not gated:
        z = skip = bias = None
    names = ["x", "dt", "A", "Bm", "Cm", "skip", "z", "bias", "h0"]
    args = dict(zip(names, (x, dt, A, Bm, Cm, skip, z, bias, h0)))
    got = ref.selective_scan_grad(*args.values(), n, dy, dh)
    for name, g in zip(names, got):
        if args[name] is None:
            continue

        def both(v, name=name):
            y, h = ref.selective_scan(**{**args, name: v}, lengths=n)[:2]
            return np.concatenate([y.ravel(), h.ravel()])
        np.testing.assert_allclose(g, differences(both, args[name], np.concatenate([dy.ravel(), dh.ravel()])), **TOL,
                                   err_msg=name)


def test_selective_scan_of_constant_steps():
    """Equal steps: the state is a geometric sum."""
    T, A, v, x = 9, -0.7, 0.3, 1.5
    one = np.ones((1, T, 1))
    y, h = ref.selective_scan(x * one, v * one, np.array([[A]]), one, 2 * one, None, None, None, None, None)[:2]
    d = np.log(1 + np.exp(v))
    a = np.exp(d * A)
    want = d * x * (1 - a ** np.arange(1, T + 1)) / (1 - a)
    np.testing.assert_allclose(y[0, :, 0], 2 * want, rtol=1e-12)
    np.testing.assert_allclose(h[0, 0, 0], want[-1], rtol=1e-12)


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("K", [1, 2, 4])
@pytest.mark.parametrize("lengths", [None, [6, 0, 1, 2]])
def test_causal_conv_gradients_match_differences(K, lengths, silu):
    rng = np.random.default_rng(K)
    B, T, D = 4, 6, 2
    x, dy = rng.standard_normal((2, B, T, D))
    state, dlast = rng.standard_normal((2, B, K - 1, D))
    names = ["x", "w", "bias", "state"]
    args = dict(zip(names, (x, rng.standard_normal((K, D)), rng.standard_normal(D), state)))
    n = None if lengths is None else np.array(lengths)
    got = ref.causal_conv_grad(*args.values(), n, silu, dy, dlast)
    for name, g in zip(names, got):
        def both(v, name=name):
            y, last = ref.causal_conv(**{**args, name: v}, lengths=n, silu=silu)[:2]
            return np.concatenate([y.ravel(), last.ravel()])
        np.testing.assert_allclose(g, differences(both, args[name], np.concatenate([dy.ravel(), dlast.ravel()])), **TOL,
                                   err_msg=name)


def test_causal_conv_is_a_convolution():
    rng = np.random.default_rng(3)
    x, w = rng.standard_normal((1, 20, 1)), rng.standard_normal((4, 1))
    y = ref.causal_conv(x, w, None, None, None, False)[0]
    np.testing.assert_allclose(y[0, :, 0], np.convolve(x[0, :, 0], w[::-1, 0])[:20], rtol=1e-12, atol=1e-14)
