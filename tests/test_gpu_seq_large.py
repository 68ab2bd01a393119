"""Sequence operators on the GPU with more workgroups than one row of a launch
holds, against 64-bit forms on the device.  Tolerances as in test_gpu_seq: U per
operation, sums of n terms n U of the terms' magnitudes, half a unit of the
output's type."""
import pytest
import torch

from gpu_util import say
from paper_2003_02989_amd import seq
from test_gpu_seq import K_SCAN, TYPES, U

pytestmark = pytest.mark.gpu
ROW = 1 << 21  # workgroups of a launch along x


def near(name, got, want, tol):
    assert torch.isfinite(got).all(), name
    over = ((got.double() - want).abs() / tol).max()
    say(f"{name}: {float(over):.3f} of the tolerance")
    assert float(over) <= 1, name


def test_embed_of_many_ids():
    N, V, D = 16 * ROW + 37, 50, 257  # sixteen rows to a workgroup
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    tok = torch.randint(-1, V + 1, (N,), device="cuda", generator=gen)
    table = torch.randn((V, D), device="cuda", generator=gen).bfloat16()
    out = seq.embed(tok, table)
    rows = torch.cat((table, torch.zeros((1, D), device="cuda", dtype=table.dtype)))
    at = torch.where((tok >= 0) & (tok < V), tok, torch.full_like(tok, V))
    for i in range(0, N, 1 << 22):
        assert torch.equal(out[i:i + (1 << 22)], rows[at[i:i + (1 << 22)]])


@pytest.mark.parametrize("ty,B,T,D", [("bf16", 4 * ROW + 3, 33, 1), ("f32", ROW + 1, 140, 1), ("f16", ROW + 5, 9, 1025)])
def test_gated_scan_of_many_records(ty, B, T, D):
    """One segment, two segments by ticket, and few steps of many channels."""
    dtype, u, tiny = TYPES[ty]
    if T == 9:
        B = B // 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    x = torch.randn((B, T, D), device="cuda", generator=gen, dtype=torch.float32).to(dtype)
    g = torch.randn((B, T, D), device="cuda", generator=gen, dtype=torch.float32).clamp_(-6, 6).to(dtype)
    dy = torch.randn((B, T, D), device="cuda", generator=gen, dtype=torch.float32).to(dtype)
    n = torch.randint(0, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
    n[:5] = torch.tensor([0, 1, T, T, T - 1], dtype=torch.int32, device="cuda")
    n[-2:] = T
    y, h, states = seq.gated_scan(x, g, lengths=n, keep=True)
    dx, dg, dh0 = seq.gated_scan_grad(x, g, states, dy, lengths=n)
    # the first and the last records, and some between
    at = torch.cat((torch.arange(300), torch.randint(0, B, (2000,), generator=torch.Generator().manual_seed(3)),
                    torch.arange(B - 300, B))).cuda()
    f = K_SCAN * min(T + 8, 500) * U
    xs, gs, ds, ns = x[at].double(), g[at].double(), dy[at].double(), n[at]
    a = torch.sigmoid(gs)
    s, m, before, mag = torch.zeros_like(xs[:, 0]), torch.zeros_like(xs[:, 0]), [], []
    for t in range(T):
        on = (t < ns)[:, None]
        before.append(s)
        new, mnew = a[:, t] * s + (1 - a[:, t]) * xs[:, t], a[:, t] * m + (1 - a[:, t]) * xs[:, t].abs()
        s, m = torch.where(on, new, s), torch.where(on, mnew, m)
        want = torch.where(on, new, 0.0)
        near("y", y[at, t], want, u * want.abs() + f * (m + 1e-30) + tiny)
        mag.append(m)
    near("h_last", h[at], s, (f + U) * (m + 1e-30))
    r, rm = torch.zeros_like(s), torch.zeros_like(s)
    for t in range(T - 1, -1, -1):
        on = (t < ns)[:, None]
        lam, lm, c = ds[:, t] + r, ds[:, t].abs() + rm, 1 - a[:, t]
        wx = torch.where(on, c * lam, 0.0)
        wg = torch.where(on, a[:, t] * c * (before[t] - xs[:, t]) * lam, 0.0)
        prev = mag[t - 1] if t else torch.zeros_like(m)
        near("dx", dx[at, t], wx, u * wx.abs() + f * lm + tiny)
        near("dg", dg[at, t], wg, u * wg.abs() + 2 * f * (prev + xs[:, t].abs()) * lm + tiny)
        r, rm = torch.where(on, a[:, t] * lam, r), torch.where(on, a[:, t] * lm, rm)
    near("dh0", dh0[at], r, (f + U) * (rm + 1e-30))


def test_layer_norm_gradient_of_the_widest_rows():
    N, D = 2, 32 * ROW + 69  # 32 columns of both sums to a workgroup
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    x, dy = (torch.randn((N, D), device="cuda", generator=gen).bfloat16() for _ in range(2))
    w = torch.ones(D, device="cuda", dtype=torch.bfloat16)
    y, mean, rstd = seq.layer_norm(x, w, keep=True)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    near("y", y, xh, 2.0 ** -8 * xh.abs() + 8 * U * (1 + xh.abs()))
    dx, dw, db = seq.layer_norm_grad(x, w, mean, rstd, dy)
    want = (dy.double() * xh).sum(0)
    near("dweight", dw, want, 2.0 ** -8 * want.abs() + 16 * U * (dy.double().abs() * (1 + xh.abs())).sum(0) + 1e-30)
    want = dy.double().sum(0)
    near("dbias", db, want, 2.0 ** -8 * want.abs() + 4 * U * dy.double().abs().sum(0) + 1e-30)


def test_cross_entropy_of_a_large_vocabulary():
    """More rows of weights to lay out than a launch holds along x."""
    N, V, D = 100, 32 * ROW + 3, 32
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    W = torch.randn((V, D), device="cuda", generator=gen, dtype=torch.bfloat16)
    h = (0.5 * torch.randn((N, D), device="cuda", generator=gen)).bfloat16()
    t = torch.randint(0, V, (N,), device="cuda", generator=gen)
    t[0], t[1], t[2] = V - 1, -1, V
    loss, lse = seq.softmax_xent(h, W, t)
    parts, top, size = [], 0.0, 0.0
    for v in range(0, V, 1 << 21):
        w = W[v:v + (1 << 21)].double()
        z = h.double() @ w.t()
        parts.append(torch.logsumexp(z, 1))
        top = max(top, float(z.abs().max()))
        size = max(size, float((h.double().abs() @ w.abs().t()).max()))
    want = torch.logsumexp(torch.stack(parts), 0)
    # a lane adds the sums of a 64th of the tiles of 128 words
    tol = D * U * size + (V // 128 // 64 + 200) * U + 8 * U * top
    near("lse", lse, want, torch.full_like(want, tol))
    ok = (t >= 0) & (t < V)
    zt = (h.double() * W[torch.where(ok, t, 0)].double()).sum(1)
    near("loss", loss, torch.where(ok, want - zt, 0.0), torch.full_like(want, 2 * tol))


def test_cross_entropy_gradient_of_many_tokens():
    """More tokens than a launch has workgroups along x, the vocabulary in two pieces."""
    N, V, D = 8 * ROW + 3, 300, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    W = torch.randn((V, D), device="cuda", generator=gen).bfloat16()
    h = torch.randn((N, D), device="cuda", generator=gen).bfloat16()
    t = torch.randint(-1, V + 1, (N,), device="cuda", generator=gen)
    # few tokens count: the bound of a sum is that of its terms that are not zero
    at = torch.cat((torch.arange(100), torch.randint(0, N, (2000,), generator=torch.Generator().manual_seed(7)),
                    torch.arange(N - 100, N))).unique().cuda()
    up = torch.zeros(N, device="cuda")
    up[at] = 1.0
    dh, dW, loss, lse = seq.softmax_xent_grad(h, W, t, up)
    hs, ts = h[at].double(), t[at]
    z = hs @ W.double().t()
    want, ok = torch.logsumexp(z, 1), (ts >= 0) & (ts < V)
    tol = D * U * float((hs.abs() @ W.double().abs().t()).max()) + (V + 32) * U + 8 * U * float(z.abs().max())
    near("lse", lse[at], want, torch.full_like(want, tol))
    p = torch.softmax(z, 1)
    p[ok.nonzero()[:, 0], ts[ok]] -= 1
    p[~ok] = 0
    u = 2.0 ** -8
    pe = p.abs() * u + tol + 2.0 ** -38  # p is stored in 16 bits
    wd = p @ W.double()
    near("dhidden", dh[at], wd, u * wd.abs() + (1 + u) * (pe @ W.double().abs()) + 2.0 ** -133)
    wd = p.t() @ hs
    near("dweight", dW, wd, u * wd.abs() + (1 + u) * (pe.t() @ hs.abs() + len(at) * U * (p.abs().t() @ hs.abs())) + 2.0 ** -133)
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert int((dh[rest] != 0).sum()) == 0
