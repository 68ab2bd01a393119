"""Plain 64-bit forms of the sequence operators (test infrastructure only).

Written from the definitions, step by step, in float64 numpy; every function
that the tests compare rounded results with also returns a magnitude: the same
sums with the absolute values of their terms, which rounding errors scale with.
"""
import numpy as np


def embed(tokens, table, scale):
    t = np.asarray(tokens).ravel()
    out = np.zeros((t.size, table.shape[1]))
    ok = (t >= 0) & (t < table.shape[0])
    out[ok] = table[t[ok]] * scale
    return out


def embed_grad(tokens, grad_out, V, scale):
    """(gradient, sum of magnitudes, number of terms)"""
    t = np.asarray(tokens).ravel()
    g, m, n = np.zeros((V, grad_out.shape[1])), np.zeros((V, grad_out.shape[1])), np.zeros(V)
    for i, v in enumerate(t):
        if 0 <= v < V:
            g[v] += scale * grad_out[i]
            m[v] += abs(scale) * np.abs(grad_out[i])
            n[v] += 1
    return g, m, n


def _sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1 / (1 + e), e / (1 + e))


def scan(x, g, h0, lengths):
    """(y, h_last, states before each step, magnitudes of y and h_last)"""
    B, T, D = x.shape
    h = np.zeros((B, D)) if h0 is None else h0.copy()
    m = np.abs(h)
    y, ym, before = np.zeros((B, T, D)), np.zeros((B, T, D)), np.zeros((B, T, D))
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    for t in range(T):
        on = (t < n)[:, None]
        with np.errstate(invalid="ignore"):
            a, c = _sigmoid(g[:, t]), _sigmoid(-g[:, t])
            before[:, t] = h
            h = np.where(on, a * h + c * x[:, t], h)
            m = np.where(on, a * m + c * np.abs(x[:, t]), m)
        y[:, t] = np.where(on, h, 0)
        ym[:, t] = np.where(on, m, 0)
    return y, h, before, ym, m


def scan_grad(x, g, h0, lengths, dy, dh_last):
    """(dx, dg, dh0, and their magnitudes)"""
    B, T, D = x.shape
    _, _, before, ym, _ = scan(x, g, h0, lengths)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    r = np.zeros((B, D)) if dh_last is None else dh_last.copy()
    rm = np.abs(r)
    dx, dg, dxm, dgm = (np.zeros((B, T, D)) for _ in range(4))
    hm = np.zeros((B, D)) if h0 is None else np.abs(h0)
    for t in range(T - 1, -1, -1):
        on = (t < n)[:, None]
        with np.errstate(invalid="ignore"):
            a, c = _sigmoid(g[:, t]), _sigmoid(-g[:, t])
            lam, lm = dy[:, t] + r, np.abs(dy[:, t]) + rm
            prev = ym[:, t - 1] if t else hm
            dx[:, t], dxm[:, t] = np.where(on, c * lam, 0), np.where(on, c * lm, 0)
            dg[:, t] = np.where(on, a * c * (before[:, t] - x[:, t]) * lam, 0)
            dgm[:, t] = np.where(on, a * c * (prev + np.abs(x[:, t])) * lm, 0)
            r, rm = np.where(on, a * lam, r), np.where(on, a * lm, rm)
    return dx, dg, r, dxm, dgm, rm


def norm(x, w, b, eps):
    """(y, mean, rstd)"""
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None] * w
    return (y if b is None else y + b), mean, rstd


def norm_grad(x, w, eps, dy):
    """(dx, dweight, dbias)"""
    _, mean, rstd = norm(x, w, None, eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    u = dy * w
    dx = rstd[:, None] * (u - u.mean(1)[:, None] - xh * (u * xh).mean(1)[:, None])
    return dx, (dy * xh).sum(0), dy.sum(0)


def xent(h, W, targets):
    """(loss, lse, logits)"""
    z = h @ W.T
    top = z.max(1, keepdims=True)
    lse = np.log(np.exp(z - top).sum(1)) + top[:, 0]
    ok = (targets >= 0) & (targets < W.shape[0])
    loss = np.where(ok, lse - z[np.arange(len(z)), np.where(ok, targets, 0)], 0)
    return loss, lse, z


def xent_grad(h, W, targets, up):
    """(dhidden, dweight, loss, lse, upstream p)"""
    loss, lse, z = xent(h, W, targets)
    p = np.exp(z - lse[:, None])
    ok = (targets >= 0) & (targets < W.shape[0])
    p[np.nonzero(ok)[0], targets[ok]] -= 1
    p = p * np.where(ok, up, 0)[:, None]
    p[~ok] = 0
    hz = np.where(ok[:, None], h, 0)
    return p @ W, p.T @ hz, loss, lse, p
