"""Plain 64-bit forms of the operators of selective models (test infrastructure
only), written from the definitions, step by step, in float64 numpy.

Functions whose results the tests compare with rounded ones also return
magnitudes: the same sums with the absolute values of their terms, which rounding
errors scale with.
"""
import numpy as np


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1 / (1 + e), e / (1 + e))


def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def _count(lengths, B, T):
    return np.full(B, T) if lengths is None else np.clip(lengths, 0, T)


def selective_scan(x, dt, A, Bm, Cm, skip, z, bias, h0, lengths):
    """y, h_last, p (y before its gate), all states [B, T + 1, D, S] (first: h0;
    past the length: kept), and (pm, pe, m, e): the magnitudes of p and of the
    states, and bounds of their errors in units of one rounding in 32 bits.

    With v = dt + bias rounded once, d = softplus(v) is off by |v| + 16 units (the
    exponential, two reciprocals, the series), the exponent d A by 4 more; the decay
    is off by |d A| times that and by 2 units of its own, a step's sum by one."""
    B, T, D = x.shape
    S = A.shape[1]
    n = _count(lengths, B, T)
    zero = np.zeros(D)
    skip = zero if skip is None else skip
    bias = zero if bias is None else bias
    h = np.zeros((B, T + 1, D, S))
    m, e = np.zeros_like(h), np.zeros_like(h)
    if h0 is not None:
        h[:, 0], m[:, 0] = h0, np.abs(h0)
    y, p, pm, pe = (np.zeros((B, T, D)) for _ in range(4))
    for b in range(B):
        for t in range(T):
            if t >= n[b]:
                h[b, t + 1], m[b, t + 1], e[b, t + 1] = h[b, t], m[b, t], e[b, t]
                continue
            v = dt[b, t] + bias
            d, off = softplus(v), np.abs(v) + 20
            a = np.exp(d[:, None] * A)
            u = (d * x[b, t])[:, None] * Bm[b, t]
            h[b, t + 1] = a * h[b, t] + u
            m[b, t + 1] = a * m[b, t] + np.abs(u)
            e[b, t + 1] = a * (e[b, t] + (3 + (off * d)[:, None] * np.abs(A)) * m[b, t]) + (3 + off)[:, None] * np.abs(u)
            p[b, t] = (Cm[b, t] * h[b, t + 1]).sum(-1) + skip * x[b, t]
            pm[b, t] = (np.abs(Cm[b, t]) * m[b, t + 1]).sum(-1) + np.abs(skip * x[b, t])
            pe[b, t] = (np.abs(Cm[b, t]) * e[b, t + 1]).sum(-1) + (S + 2) * pm[b, t]
            y[b, t] = p[b, t] * (1 if z is None else z[b, t] * sigmoid(z[b, t]))
    return y, h[:, T], p, h, (pm, pe, m, e)


def selective_scan_grad(x, dt, A, Bm, Cm, skip, z, bias, h0, lengths, dy, dh_last, absolute=False):
    """dx, ddt, dA, dB, dC, dskip, dz, ddt_bias, dh0.  With `absolute` every term
    counts with its magnitude instead: what the errors of the sums scale with."""
    f = np.abs if absolute else lambda v: v
    B, T, D = x.shape
    S = A.shape[1]
    n = _count(lengths, B, T)
    zero = np.zeros(D)
    skip_, bias_ = zero if skip is None else skip, zero if bias is None else bias
    _, _, p, h, (pm, _, m, _) = selective_scan(x, dt, A, Bm, Cm, skip, z, bias, h0, lengths)
    if absolute:
        h, p = m, pm
    dx, ddt, dz = (np.zeros((B, T, D)) for _ in range(3))
    dB, dC = np.zeros((B, T, S)), np.zeros((B, T, S))
    dA, dskip, dbias, dh0 = np.zeros((D, S)), np.zeros(D), np.zeros(D), np.zeros((B, D, S))
    for b in range(B):
        r = np.zeros((D, S)) if dh_last is None else f(dh_last[b])
        for t in range(n[b] - 1, -1, -1):
            v = dt[b, t] + bias_
            d, sg = softplus(v), sigmoid(v)
            a = np.exp(d[:, None] * A)
            xt, Bt, Ct = f(x[b, t]), f(Bm[b, t]), f(Cm[b, t])
            q = f(dy[b, t])
            if z is not None:
                s = sigmoid(z[b, t])
                # silu' is a sum of two terms, which cancel near z = -1.28
                dz[b, t] = f(dy[b, t]) * p[b, t] * (s + f(z[b, t]) * s * (1 - s))
                q = q * f(z[b, t] * s)
            l = q[:, None] * Ct + r
            dC[b, t] = (q[:, None] * h[b, t + 1]).sum(0)
            dB[b, t] = ((d * xt)[:, None] * l).sum(0)
            bl = (Bt * l).sum(-1)
            dx[b, t] = d * bl + f(skip_) * q
            w = a * h[b, t] * l
            ddt[b, t] = ((f(A) * w).sum(-1) + xt * bl) * sg
            dA += d[:, None] * w
            dskip += q * xt
            dbias += ddt[b, t]
            r = a * l
        dh0[b] = r
    return dx, ddt, dA, dB, dC, dskip, dz, dbias, dh0


def causal_conv(x, w, bias, state, lengths, silu):
    """y, last, u (y before silu) and u's magnitude"""
    B, T, D = x.shape
    K = w.shape[0]
    n = _count(lengths, B, T)
    y, u, um = (np.zeros((B, T, D)) for _ in range(3))
    last = np.zeros((B, K - 1, D))
    for b in range(B):
        xs = np.concatenate([np.zeros((K - 1, D)) if state is None else state[b], x[b, :n[b]]])
        last[b] = xs[n[b]:]
        for t in range(n[b]):
            terms = w * xs[t:t + K]
            u[b, t] = terms.sum(0) + (0 if bias is None else bias)
            um[b, t] = np.abs(terms).sum(0) + (0 if bias is None else np.abs(bias))
            y[b, t] = u[b, t] * sigmoid(u[b, t]) if silu else u[b, t]
    return y, last, u, um


def causal_conv_grad(x, w, bias, state, lengths, silu, dy, dlast, absolute=False):
    """dx, dweight, dbias, dstate.  With `absolute` every term counts with its
    magnitude; an error of u's sum moves silu' by at most half of it (|silu''| <=
    1/2), so that K units of u's magnitude count beside silu's own terms."""
    f = np.abs if absolute else lambda v: v
    B, T, D = x.shape
    K = w.shape[0]
    n = _count(lengths, B, T)
    _, _, u, um = causal_conv(x, w, bias, state, lengths, silu)
    dx, dw, db, ds = np.zeros((B, T, D)), np.zeros((K, D)), np.zeros(D), np.zeros((B, K - 1, D))
    for b in range(B):
        xs = np.concatenate([np.zeros((K - 1, D)) if state is None else state[b], x[b, :n[b]]])
        back = np.zeros_like(xs)
        if dlast is not None:
            back[n[b]:] += f(dlast[b])
        for t in range(n[b]):
            s = sigmoid(u[b, t])
            slope = s + f(u[b, t]) * s * (1 - s) + (um[b, t] if absolute else 0) if silu else 1
            g = f(dy[b, t]) * slope
            for k in range(K):
                back[t + k] += f(w[k]) * g
                dw[k] += g * f(xs[t + k])
            db += g
        ds[b], dx[b, :n[b]] = back[:K - 1], back[K - 1:]
    return dx, dw, db, ds


def beam_candidates(logits, scores, last=None, end=None):
    """The scores [R, W, V] of all candidates."""
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = logits.max(-1, keepdims=True)
        top = np.where(np.isfinite(top), top, 0)
        lse = np.log(np.exp(logits - top).sum(-1, keepdims=True)) + top
        c = scores[..., None] + (logits - lse)
    if last is not None:
        on = last == end
        c[on] = -np.inf
        c[..., end] = np.where(on, scores, c[..., end])
    return np.where(c < np.inf, c, -np.inf)


def beam_select(logits, scores, K, last=None, end=None):
    """scores, parents and tokens [R, K] of the best candidates, by plain sorting:
    score, then beam, then logit, then id."""
    R, W, V = logits.shape
    c = beam_candidates(logits, scores, last, end)
    out = [np.zeros((R, K)), np.zeros((R, K), int), np.zeros((R, K), int)]
    beam, word = np.divmod(np.arange(W * V), V)
    for r in range(R):
        flat = c[r].ravel()
        # where nothing but the id is left to tell candidates apart
        logit = np.where(flat > -np.inf, logits[r].ravel(), 0)
        order = np.lexsort((word, -logit, beam, -flat))[:K]
        out[0][r], out[1][r], out[2][r] = flat[order], beam[order], word[order]
    return out
