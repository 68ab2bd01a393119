"""Sequence operators on the GPU at sizes where another variant takes over,
against the oracle's 64-bit forms, with the tolerances of test_gpu_seq."""
import numpy as np
import pytest
import torch

import test_gpu_seq as base
from gpu_util import say
from oracle import seq as ref
from paper_2003_02989_amd import seq
from test_gpu_seq import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("kind", ["uniform", "one"])
@pytest.mark.parametrize("N,V,D", [(48, 17, 4096), (63, 3, 2049), (57, 5, 2100), (33, 9, 4099), (16, 17, 8193),
                                   (64, 3, 2100), (65, 3, 2100), (66, 3, 2100)])
def test_table_gradient_of_few_wide_rows(ty, kind, N, V, D):
    """Too wide for the kernel of few ids, too few ids for a long run."""
    base.test_embed_grad(ty, N, V, D, kind)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N,D,pad", [(3, 4097, 0), (5, 5001, 2), (2, 8191, 1), (7, 8192, 0), (3, 8193, 0), (4, 12001, 3),
                                     (2, 16383, 1), (5, 16384, 0), (4100, 8200, 0)])
def test_layer_norm_of_rows_that_a_whole_workgroup_holds(ty, N, D, pad):
    base.test_layer_norm_and_gradients(ty, True, N, D, pad)


@pytest.mark.parametrize("ty", TYPES)
def test_cross_entropy_of_nothing(ty):
    """No tokens and no vocabulary: empty results."""
    dtype = TYPES[ty][0]
    e = torch.zeros((0, 5), dtype=dtype, device="cuda")
    t, up = torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    dh, dW, loss, lse = seq.softmax_xent_grad(e, e, t, up)
    assert dh.shape == dW.shape == (0, 5) and loss.shape == lse.shape == (0,)
    assert seq.softmax_xent(e, e, t)[0].shape == (0,)


@pytest.mark.parametrize("ty", TYPES)
@pytest.mark.parametrize("N", [16, 17, 40, 64, 65])
@pytest.mark.parametrize("ld,shift", [(129, 0), (136, 0), (136, 1), (128, 0)])
def test_cross_entropy_of_weights_that_lie_anywhere(ty, N, ld, shift):
    """Whole pieces of D = 128 elements in rows that are aligned or not."""
    dtype = TYPES[ty][0]
    rng = np.random.default_rng(N)
    V, D = 300, 128
    h, hv = base.put(rng.standard_normal((N, D)), dtype)
    W, Wv = base.put(0.2 * rng.standard_normal((V, ld)), dtype)
    room = torch.empty(V * ld + 8, dtype=dtype, device="cuda")[shift:shift + V * ld].view(V, ld)
    room.copy_(W)
    t = rng.integers(-1, V + 1, N)
    loss, lse = seq.softmax_xent(h, room[:, :D], torch.as_tensor(t).cuda())
    wl, ws, z = ref.xent(hv, Wv[:, :D], t)
    es = base.logit_error(ty, hv, Wv[:, :D]).max(1) + (V + 32) * base.U + 4 * base.U * np.abs(z).max(1)
    base.check("lse", lse, ws, es)
    base.check("loss", loss, wl, np.where((t >= 0) & (t < V), 2 * es, 0))


@pytest.mark.parametrize("ty", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["equal", "powers of two", "any", "signs and zeros", "two classes"])
@pytest.mark.parametrize("N,V,D", [(600, 4097, 64), (1000, 4097, 130)])
def test_cross_entropy_gradient_of_unequal_tokens(ty, kind, N, V, D):
    """dweight loses nothing to upstream: its error is that of its own rounding and
    of p's.  With u half a unit of 1, rounding numbers of any digits costs 0.42 u in
    the mean square, and p just below 1 is off by u / 2 / sqrt(3) = 0.29 u: together
    1.21 times the former at most.  A further rounding of any digits makes it 1.41
    at least."""
    dtype = TYPES[ty][0]
    rng = np.random.default_rng(N)
    h, hv = base.put(rng.standard_normal((N, D)), dtype)
    W, Wv = base.put(1.5 / np.sqrt(D) * rng.standard_normal((V, D)), dtype)
    t = rng.integers(0, V, N)
    up = {"equal": np.full(N, 0.7), "powers of two": 0.7 * 2.0 ** -rng.integers(0, 9, N), "any": rng.random(N) + 0.02,
          "signs and zeros": rng.standard_normal(N) * (rng.random(N) < 0.8),
          "two classes": np.where(rng.random(N) < 0.5, 1.0, 0.37)}[kind]
    up, upv = base.put(up, torch.float32)
    dh, dW, _, _ = seq.softmax_xent_grad(h, W, torch.as_tensor(t).cuda(), up)
    wdh, wdW, _, _, _ = ref.xent_grad(hv, Wv, t, upv)
    for name, got, want in (("dhidden", dh, wdh), ("dweight", dW, wdW)):
        least = np.linalg.norm(torch.as_tensor(want).to(dtype).double().numpy() - want)
        err = np.linalg.norm(got.double().cpu().numpy() - want)
        say(ty, kind, name, err / least)
        assert err <= 1.25 * least, name


def test_layer_norm_of_no_values():
    """Rows without columns: their mean is not a number, whatever the memory held."""
    torch.full((2, 64), 3.0, device="cuda")  # what the allocator hands out next
    y, mean, rstd = seq.layer_norm(torch.zeros((64, 0), device="cuda"), torch.zeros(0, device="cuda"), keep=True)
    assert y.shape == (64, 0) and torch.isnan(mean).all() and torch.isnan(rstd).all()
    dx, dw, db = seq.layer_norm_grad(y, torch.zeros(0, device="cuda"), mean, rstd, y)
    assert dx.shape == (64, 0) and dw.shape == db.shape == (0,)
