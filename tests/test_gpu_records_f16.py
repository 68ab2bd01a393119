"""The recurrent model of measurement records in float16: gradients of a mean over
many shots, whose terms lie below the smallest numbers of the type."""
import numpy as np
import pytest
import torch

from gpu_util import say
from paper_2003_02989_amd.records import RecordModel, ising_records
from test_gpu_records import oracle_loss

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B", [3, 4096])
def test_gradients_of_a_mean_over_many_shots(dtype, B):
    T = 32
    records = ising_records(4, T, B, seed=8)
    records[1, 3:] = -1
    model = RecordModel(4, 32, dtype=dtype, seed=9)
    loss, grads = model.loss_and_grads(records)
    wl, wg = oracle_loss(model, records, None)
    # some ten tensors between the shots and a gradient (looked-up rows, states,
    # normalised states, p, and the gradients of each), each rounded to half a unit u
    # of the type, and factors of up to four from one to the next
    u = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    assert abs(float(loss) - wl) <= 40 * u * wl
    for k, g in grads.items():
        g = g.double().cpu().numpy()
        err = np.linalg.norm(g - wg[k]) / np.linalg.norm(wg[k])
        say(str(dtype), B, k, "error", err)
        assert err <= 40 * u, k


def test_a_step_in_float16_moves_every_parameter():
    model = RecordModel(4, 32, dtype=torch.float16, seed=9)
    before = {k: p.clone() for k, p in model.params.items()}
    model.step(ising_records(4, 32, 2048, seed=8))
    for k, p in model.params.items():
        assert torch.isfinite(p).all()
        # rows of bitstrings that the shots hold: nearly all of the 17
        assert float((p != before[k]).float().mean()) > 0.5, k
