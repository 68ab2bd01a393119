"""What the sequence calls launch, recorded on the host without a GPU: no call
that the checks of arguments let through has a grid that HIP refuses."""
import os

import pytest

import launches as la

ROOT = la.ROOT


def run(calls, tmp_path):
    got, _ = la.recorded(calls, tmp_path)
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


def test_every_variant_of_layer_norm_is_reached(tmp_path):
    """Rows of every width go to the variant that their width is meant for, and
    no variant is left that no width reaches."""
    widths = sorted({max(1, w + d) for w in (1, 4, 8, 32, 64, 128, 256, 512, 1024, 2048, 4096, 8192, 16384) for d in (-1, 0, 1)})
    widths += [768, 769, 1536, 1537, 100003]
    calls = [f(ty, 5, D) for f in (la.norm, la.norm_grad) for ty in range(3) for D in widths]
    got, kernels = la.recorded(calls, tmp_path)
    assert all(g["rc"] == 0 for g in got)
    reached = {n for g in got for n in names(g)}
    assert {k for k in kernels if "k_norm" in k} == reached
    for c, g in zip(calls, got):
        if c[0] == "tq_layer_norm":
            one = 4096 if c[3] == 0 else 8192  # of 16 pieces to a lane of 256, in registers
            want = "Li256ELi4E" if one // 2 < c[5] <= one else "Li1024ELi2E" if one < c[5] <= 2 * one else "k_norm_wide" if c[5] > 2 * one else ""
            assert want in names(g)[0], (c[3], c[5], names(g))


def test_sizes_of_nothing(tmp_path):
    """Every size that may be zero, alone and together: the workspace is asked
    for and the call made; none ends the process, none has an empty grid."""
    calls = []
    for ty in range(3):
        for N in (0, 1, 70):
            for V in (0, 1, 300):
                for D in (0, 1, 64):
                    if not (N and not V):
                        calls += [("tq_softmax_xent_workspace", ty, N, V, D), la.xent(ty, N, V, D),
                                  ("tq_softmax_xent_grad_workspace", ty, N, V, D), la.xent_grad(ty, N, V, D)]
                    calls += [("tq_embed_grad_workspace", V, D, N), la.embed(ty, N, V, D), la.embed_grad(ty, N, V, D)]
                calls += [("tq_layer_norm_grad_workspace", N, V), la.norm(ty, N, V), la.norm_grad(ty, N, V)]
                for B in (0, 2):
                    calls += [("tq_gated_scan_workspace", B, N, V), la.scan(ty, B, N, V), la.scan_grad(ty, B, N, V)]
    run(calls, tmp_path)


M31 = (1 << 31) - 1


def test_largest_sizes(tmp_path):
    """Sizes up to the limits that the header names are launched, or refused
    before anything is: as unsupported, by the checks of the arguments."""
    calls = []
    for ty in range(3):
        calls += [la.embed(ty, M31, V, D) for V in (5, M31) for D in (1, 64, 65, 2048)]
        calls += [la.embed_grad(ty, N, V, D) for N in (100, 600, M31) for V in (5, M31) for D in (1, 300, 1 << 20)]
        for B, T, D in ((M31, 1, 1), (M31, 64, 1), (1 << 23, 33, 1), (1 << 23, 64, 130), (1, M31, 1), (1, M31, 4000),
                        (1 << 16, 1, 1 << 20), (1 << 16, 8, 1 << 20), (1 << 14, 16, 1 << 20), (1 << 26, 1000, 3)):
            calls += [la.scan(ty, B, T, D), la.scan_grad(ty, B, T, D)]
        calls += [f(ty, N, D) for f in (la.norm, la.norm_grad)
                  for N, D in ((M31, 1), (M31, 64), (M31, 100003), (1, M31), (5000, M31), (1 << 22, 16385))]
        for N, V, D in ((M31, 16, 1), (M31, 16, 64), (4, M31, 64), (60, M31, 64), (100, M31, 33), (100, M31, 64),
                        (1 << 20, 1 << 20, 64), (1 << 24, 300, 8), (1 << 24, 300, 64), (100, 1 << 26, 32), (1 << 14, 5, 1 << 20)):
            calls += [la.xent(ty, N, V, D), la.xent_grad(ty, N, V, D)]
        calls += [la.xent_grad(ty, 0, M31, 64)]
    run(calls, tmp_path)
    # too many tiles for one launch
    for c in (la.xent(0, M31, M31, 8), la.xent_grad(1, M31, 5, 1 << 20), la.xent_grad(1, 5, M31, 1 << 20),
              la.scan(1, M31, 65, 1), la.scan_grad(0, M31, 64, 65)):
        got = la.recorded([c], tmp_path)[0][0]
        assert got["rc"] == 2 and not got["kernels"], (c[0], c[1:8], got["rc"], got["error"])


def test_few_tokens_do_not_copy_the_weights(tmp_path):
    """Losses of up to 64 tokens read the weights where they are, however these lie."""
    calls = [la.xent(ty, N, 65537, D, ld) for ty in range(3) for N in (1, 16, 17, 40, 64)
             for D, ld in ((512, 512), (512, 513), (512, 516), (500, 500), (64, 65))]
    # weights that begin inside a 16-byte piece
    calls += [c[:7] + (la.P + 2,) + c[8:] for c in calls if c[3] != 0]
    for c, g in zip(calls, run(calls, tmp_path)):
        assert not any("k_lay_weight" in n for n in names(g)), (c[3:6], c[2], c[7], names(g))
