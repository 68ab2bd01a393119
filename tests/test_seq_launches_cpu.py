"""What the sequence calls launch, recorded on the host without a GPU: no call
that the checks of arguments let through has a grid that HIP refuses."""
import os

import pytest

import launches as la

ROOT = la.ROOT


def run(calls, tmp_path):
    got = la.recorded(calls, tmp_path)
    for c, g in zip(calls, got):
        assert g["rc"] == 0, (c[0], c[1:8], g["error"], g["kernels"][-3:])
    return got


def names(answer):
    return [k[0] for k in answer["kernels"]]


@pytest.mark.parametrize("ty", [0, 1, 2])
def test_table_gradient_of_any_number_of_ids(ty, tmp_path):
    """No id, few and many, of narrow and wide rows: the join of long runs is
    launched only where a run can be long."""
    calls = [la.embed_grad(ty, N, 17, D) for D in (1, 64, 257, 600, 2049, 2100, 4096, 8193, 1 << 20)
             for N in (0, 1, 15, 16, 33, 48, 56, 57, 63, 64, 65, 129, 512, 513, 4097)]
    for c, g in zip(calls, run(calls, tmp_path)):
        joins = [n for n in names(g) if "k_embed_join" in n]
        assert not joins or c[7] > 64, c[:8]
