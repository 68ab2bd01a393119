"""The 64-bit sequence operators of the oracle: gradients against central
differences, and closed forms."""
import numpy as np
import pytest

from oracle import seq as ref


def differences(f, x, up, eps=1e-6):
    """Gradient of sum(up * f(x)) by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += eps
        b[i] -= eps
        g[i] = ((f(a) - f(b)) * up).sum() / (2 * eps)
    return g


# central differences in float64: truncation eps^2 times third derivatives of
# order one (1e-12), rounding 1e-16 / eps times values of order ten (1e-9)
TOL = dict(rtol=1e-6, atol=2e-8)


def test_embed_grad_is_the_transpose_of_embed():
    rng = np.random.default_rng(1)
    t = np.array([3, -1, 0, 3, 7, 5])
    table, up = rng.standard_normal((7, 3)), rng.standard_normal((6, 3))
    d = differences(lambda w: ref.embed(t, w, 1.7), table, up)
    np.testing.assert_allclose(ref.embed_grad(t, up, 7, 1.7)[0], d, **TOL)
    assert np.all(ref.embed(t, table, 1.7)[[1, 4]] == 0)


@pytest.mark.parametrize("lengths", [None, [5, 0, 2]])
def test_scan_gradients_match_differences(lengths):
    rng = np.random.default_rng(2)
    B, T, D = 3, 5, 2
    x, g, dy = (rng.standard_normal((B, T, D)) for _ in range(3))
    h0, dh = rng.standard_normal((B, D)), rng.standard_normal((B, D))
    n = None if lengths is None else np.array(lengths)
    dx, dg, dh0 = ref.scan_grad(x, g, h0, n, dy, dh)[:3]

    def out(x, g, h0):
        y, h = ref.scan(x, g, h0, n)[:2]
        return np.concatenate([y, h[:, None]], 1)
    up = np.concatenate([dy, dh[:, None]], 1)
    np.testing.assert_allclose(dx, differences(lambda v: out(v, g, h0), x, up), **TOL)
    np.testing.assert_allclose(dg, differences(lambda v: out(x, v, h0), g, up), **TOL)
    np.testing.assert_allclose(dh0, differences(lambda v: out(x, g, v), h0, up), **TOL)


def test_scan_with_a_constant_gate_is_a_geometric_sum():
    T = 9
    y = ref.scan(np.ones((1, T, 1)), np.zeros((1, T, 1)), np.zeros((1, 1)), None)[0]
    np.testing.assert_allclose(y[0, :, 0], 1 - 0.5 ** np.arange(1, T + 1), rtol=1e-14)


def test_norm_gradients_match_differences():
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((4, 6)), rng.standard_normal((4, 6))
    w, b = rng.standard_normal(6), rng.standard_normal(6)
    dx, dw, db = ref.norm_grad(x, w, 1e-3, dy)
    np.testing.assert_allclose(dx, differences(lambda v: ref.norm(v, w, b, 1e-3)[0], x, dy), **TOL)
    np.testing.assert_allclose(dw, differences(lambda v: ref.norm(x, v, b, 1e-3)[0], w, dy), **TOL)
    np.testing.assert_allclose(db, differences(lambda v: ref.norm(x, w, v, 1e-3)[0], b, dy), **TOL)


def test_xent_gradients_match_differences():
    rng = np.random.default_rng(4)
    h, W, up = rng.standard_normal((5, 3)), rng.standard_normal((6, 3)), rng.standard_normal(5)
    t = np.array([0, 5, -1, 3, 6])
    dh, dW = ref.xent_grad(h, W, t, up)[:2]
    np.testing.assert_allclose(dh, differences(lambda v: ref.xent(v, W, t)[0], h, up), **TOL)
    np.testing.assert_allclose(dW, differences(lambda v: ref.xent(h, v, t)[0], W, up), **TOL)
    assert np.all(dh[[2, 4]] == 0)
    np.testing.assert_allclose(ref.xent(np.zeros((1, 3)), W, np.array([2]))[0], np.log(6), rtol=1e-14)
