"""The sizes of test_gpu_model_runs.py are those that they are meant to be: what
their calls launch, recorded on the host without a GPU."""
import test_gpu_model_runs as sizes
from test_model_launches_cpu import _lists, conv, conv_grad, run, scan, scan_grad  # noqa: F401 (the fixture serves here too)


def grid(call, name):
    """Workgroups of the one kernel with `name` in its name that a call launches."""
    found = [k for k in call["kernels"] if name in k[0]]
    assert len(found) == 1, call["kernels"]
    return found[0][1] * found[0][2]


def up(a, b):
    return -(-a // b)


def test_convolutions_have_long_runs(tmp_path):
    calls, want = [], []
    for ty in range(3):
        for B, T, D, K, forward, backward in sizes.CONVS:
            V, G = (4, 8, 8)[ty], 2
            V, G = V if D >= V else 1, G if D >= G else 1
            for ragged in (True, False):
                f, g = list(conv(ty, B, T, D, K)), list(conv_grad(ty, B, T, D, K))
                if not ragged:
                    f[12] = g[12] = None
                calls += [tuple(f), tuple(g)]
                runs, pieces = B * up(T, backward), up(D, G)
                rows = min(runs, (256 * 2048 if ragged else 256 * 1024) // pieces)
                want.append((up(B * up(T, forward) * up(D, V), 256), up(rows * pieces, 256)))
                assert forward > 8 and backward > 8
                if (B, T) == (8200, 1030):
                    assert runs > rows  # threads with a second run
    got, _ = run(calls, tmp_path)
    for k, (f, g) in enumerate(want):
        assert grid(got[2 * k], "k_conv") == f and grid(got[2 * k + 1], "k_conv_grad") == g, calls[2 * k][1:6]


def test_scans_have_chunks_and_workgroups_with_several_items(tmp_path):
    calls = []
    for B, T, D, S, _, ragged in sizes.EXACT:
        f, g = list(scan(0, B, T, D, S, True)), list(scan_grad(0, B, T, D, S))
        if not ragged:
            f[25] = g[25] = None
        calls += [tuple(f), tuple(g)]
    got, _ = run(calls, tmp_path)
    several = most = 0
    for k, (B, T, D, S, chunks, _) in enumerate(sizes.EXACT):
        slabs = up(D, 64)
        main = [v for v in got[2 * k]["kernels"] if "k_select" in v[0] and "chain" not in v[0]][-1]
        assert main[1] * main[2] == B * chunks * slabs, sizes.EXACT[k]
        groups = grid(got[2 * k + 1], "k_select_grad")
        assert any("k_select_back" in v[0] for v in got[2 * k + 1]["kernels"]) == (chunks > 1)
        several += B * chunks * slabs > groups
        most = max(most, chunks)
    assert several >= 6 and most > 2 * 32  # items in turn; starts of chunks read 32 together


def test_single_steps_in_fp32_take_several_records_a_thread(tmp_path):
    calls = [scan(ty, B, 1, D, S) for ty in range(3) for B, D, S in sizes.STEPS]
    got, _ = run(calls, tmp_path)
    for c, g in zip(calls, got):
        ty, B, D, S = c[1], c[2], c[4], c[5]
        lanes = 1
        while 4 * lanes < S:
            lanes *= 2
        slabs = up(D, 256 // lanes)
        assert B * slabs >= 8192 and B % 4
        assert grid(g, "k_select_step") == (up(B, 4) if ty == 0 and lanes > 1 else B) * slabs


def test_single_steps_of_more_workgroups_than_31_bits_go_by_tiles(tmp_path):
    most = (1 << 31) - 1
    got, _ = run([scan(ty, most, 1, D, S) for ty in range(3) for D, S in ((64, 64), (1, 64), (64, 4), (17, 64))], tmp_path)
    for g, step in zip(got, [False, True, True, False] * 3):
        assert [("k_select_step" in k[0]) for k in g["kernels"]] == [step], g
