"""What the calls of selective models launch, recorded on the host without a
GPU: no call that the checks of arguments let through has a grid that HIP
refuses."""
import pytest

import launches as la

P, ALL = la.P, la.ALL

# beside the kinds of launches.py: Q a list of pointers, N of int64, I of int32
la.SPECS.update({
    "tq_selective_scan_workspace": "nnnnz",
    "tq_selective_scan": "innnn" + "pnn" * 2 + "p" + "pnn" * 2 + "p" + "pnn" + "ppp" + "pnn" + "ppp" + "sp",
    "tq_selective_scan_grad_workspace": "nnnnz",
    "tq_selective_scan_grad": "innnn" + "pnn" * 2 + "p" + "pnn" * 2 + "p" + "pnn" + "ppp" + "pnn" + "p" + "pnn" * 5 + "ppppp" + "sp",
    "tq_causal_conv": "innnn" + "pnn" + "pppp" + "i" + "pnn" + "pp",
    "tq_causal_conv_grad_workspace": "nnnnz",
    "tq_causal_conv_grad": "innnn" + "pnn" + "pppp" + "i" + "pnn" + "p" + "pnn" + "pppp" + "sp",
    "tq_clip_grad_norm_workspace": "nNz",
    "tq_clip_grad_norm": "nQNIffQIppsp",
    "tq_beam_select_workspace": "innnnz",
    "tq_beam_select": "innnnpnppnppppsp",
    "tq_beam_reorder": "nQQNnnnpp",
})


@pytest.fixture(autouse=True)
def _lists(monkeypatch):
    kinds = 'kinds = {"p"'
    assert kinds in la._CHILD
    child = la._CHILD.replace(kinds, '''lists = {"Q": ctypes.c_void_p, "N": ctypes.c_int64, "I": ctypes.c_int32}
class Kinds(dict):
    def __missing__(self, k):
        return lambda a: (lists[k] * len(a))(*a)
kinds = Kinds() | {"p"''').replace("kinds = Kinds() | {", "kinds = Kinds(); kinds.update({").replace(
        '"f": ctypes.c_float}', '"f": ctypes.c_float})')
    monkeypatch.setattr(la, "_CHILD", child)


def scan(ty, B, T, D, S, keep=False):
    s, n = [T * D, D], [T * S, S]
    return ("tq_selective_scan", ty, B, T, D, S, P, *s, P, *s, P, P, *n, P, *n, P, P, *s, P, P, P, P, *s, P,
            P if keep else None, P, ALL, None)


def scan_grad(ty, B, T, D, S):
    s, n = [T * D, D], [T * S, S]
    return ("tq_selective_scan_grad", ty, B, T, D, S, P, *s, P, *s, P, P, *n, P, *n, P, P, *s, P, P, P, P, *s, P, P, *s, P, *s,
            P, *s, P, *n, P, *n, P, P, P, P, P, ALL, None)


def conv(ty, B, T, D, K):
    s = [T * D, D]
    return ("tq_causal_conv", ty, B, T, D, K, P, *s, P, P, P, P, 1, P, *s, P, None)


def conv_grad(ty, B, T, D, K):
    s = [T * D, D]
    return ("tq_causal_conv_grad", ty, B, T, D, K, P, *s, P, P, P, P, 1, P, *s, P, P, *s, P, P, P, P, ALL, None)


def clip(counts, ty=0):
    n = len(counts)
    return ("tq_clip_grad_norm", n, [P] * n, counts, [ty] * n, 1.0, 1.0, [2 * P] * n, [0] * n, P, P, ALL, None)


def beam(ty, R, W, V, K):
    return ("tq_beam_select", ty, R, W, V, K, P, V, P, P, 0, P, P, P, P, ALL, None)


def reorder(rows, R, W, K):
    n = len(rows)
    return ("tq_beam_reorder", n, [P] * n, [2 * P] * n, rows, R, W, K, P, None)


def run(calls, tmp_path):
    got, kernels = la.recorded(calls, tmp_path)
    for c, g in zip(calls, got):
        assert g["rc"] == 0, (c[0], c[1:8], g["error"], g["kernels"][-3:])
    return got, kernels


M31 = (1 << 31) - 1


def test_sizes_of_nothing(tmp_path):
    """Every size that may be zero, alone and together."""
    calls = []
    for ty in range(3):
        for B in (0, 1, 3):
            for T in (0, 1, 2, 40):
                for D in (0, 1, 70):
                    calls += [("tq_selective_scan_workspace", B, T, D, 5), ("tq_selective_scan_grad_workspace", B, T, D, 5),
                              scan(ty, B, T, D, 5), scan(ty, B, T, D, 5, True), scan_grad(ty, B, T, D, 5),
                              ("tq_causal_conv_grad_workspace", B, T, D, 3), conv(ty, B, T, D, 3), conv(ty, B, T, D, 1),
                              conv_grad(ty, B, T, D, 3), conv_grad(ty, B, T, D, 1)]
        calls += [beam(ty, 0, 1, 1, 1), beam(ty, 1, 1, 1, 1), beam(ty, 1, 64, 1, 64)]
    calls += [clip(c) for c in ([], [0], [0] * 300, [1], [0, 5, 0], [0] * 200 + [100000])]
    calls += [reorder(c, 2, 3, 3) for c in ([], [0], [0] * 300, [1])] + [reorder([8], 0, 3, 3), reorder([8], 2, 0, 3)]
    run(calls, tmp_path)


def test_largest_sizes(tmp_path):
    """Sizes up to the limits that the header names are launched."""
    calls = []
    for ty in range(3):
        for B, T, D, S in ((M31, 1, 1, 1), (M31, 1, 64, 64), (M31, 64, 1, 16), (1 << 16, 1, 1 << 20, 16), (1, M31, 1, 16),
                           (1, M31, 4000, 64), (1 << 20, 1000, 100, 17), (3, 1 << 20, 1 << 15, 5)):
            calls += [scan(ty, B, T, D, S), scan(ty, B, T, D, S, True), scan_grad(ty, B, T, D, S)]
        for B, T, D, K in (((1 << 30) - 1, 8, 2, 8), (M31, 1, 1, 2), (1 << 12, 1, 1 << 20, 4), (1, M31, 28, 4), (1, M31, 7, 8),
                           (1 << 29, 3, 9, 3), (1 << 20, 0, 8000, 4)):
            calls += [conv(ty, B, T, D, K), conv_grad(ty, B, T, D, K)]
        for R, W, V, K in ((M31, 1, 1, 1), (M31, 1, 2048, 64), (1 << 25, 63, 100, 64), (1, 1, M31, 64), (60, 64, M31 // 4, 64),
                           (1 << 22, 64, 14000, 1)):
            calls += [beam(ty, R, W, V, K)]
    calls += [clip([(1 << 40) - 1] * 5), clip([5] * 2000), clip([M31] * 101, 1)]
    calls += [reorder([1], M31, 64, 1), reorder([1 << 15] * 130, 1 << 25, 64, 60), reorder([(1 << 40) - 1] * 3, 1, 1, 1)]
    run(calls, tmp_path)


def test_scans_find_room_in_their_workspace(tmp_path):
    """With lengths and without, which are cut into chunks by different rules; a launch
    that needs more than the workspace function gives is refused."""
    calls = []
    for S in (3, 16, 40, 64):
        for B, D in ((1, 5), (1, 1000), (7, 64), (9, 300), (20, 1200), (25, 1100), (64, 512), (300, 40), (3000, 64)):
            for T in (2, 17, 64, 95, 96, 100, 350, 1200, 5000):
                for call, at in ((scan(0, B, T, D, S), 25), (scan_grad(0, B, T, D, S), 25)):
                    calls += [call, (*call[:at], None, *call[at + 1:])]
    run(calls, tmp_path)


def test_no_kernel_is_left_that_no_call_reaches(tmp_path):
    calls = []
    for ty in range(3):
        for S in (1, 5, 16, 17, 33, 64):
            for B, T, D in ((2, 1, 3), (5000, 1, 300), (2, 7, 3), (1, 3000, 3)):
                calls += [scan(ty, B, T, D, S), scan(ty, B, T, D, S, True), scan_grad(ty, B, T, D, S)]
        for K in range(1, 9):
            for T, D in ((1, 1), (9, 1), (1, 8), (9, 8)):
                calls += [conv(ty, 2, T, D, K), conv_grad(ty, 2, T, D, K)]
        calls += [beam(ty, 2, 2, V, 2) for V in (17, 1025, 30000)]
    calls += [clip([5]), clip([100000]), reorder([8], 1, 1, 1)]
    got, kernels = run(calls, tmp_path)
    reached = {k[0] for g in got for k in g["kernels"]}
    ours = {k for k in kernels if any(n in k for n in ("k_select", "k_conv", "k_clip", "k_beam"))}
    assert len(ours) > 100 and ours == reached, sorted(ours - reached)


def test_the_workspace_is_what_the_call_asks_for(tmp_path):
    """A call with the bytes that the *_workspace function gives is accepted, with
    one less refused."""
    calls, tails = [], []
    for f, need in ((scan(1, 3, 5000, 70, 16), ("tq_selective_scan_workspace", 3, 5000, 70, 16)),
                    (scan_grad(1, 3, 5000, 70, 16), ("tq_selective_scan_grad_workspace", 3, 5000, 70, 16)),
                    (conv_grad(2, 3, 500, 70, 4), ("tq_causal_conv_grad_workspace", 3, 500, 70, 4)),
                    (clip([100000, 7]), ("tq_clip_grad_norm_workspace", 2, [100000, 7])),
                    (beam(1, 3, 4, 100000, 5), ("tq_beam_select_workspace", 1, 3, 4, 100000, 5))):
        calls.append(need)
        tails.append(f)
    got, _ = run(calls, tmp_path)
    enough = [f[:-2] + (g["need"], None) for f, g in zip(tails, got)]
    less = [f[:-2] + (g["need"] - 1, None) for f, g in zip(tails, got)]
    assert all(g["need"] > 0 for g in got)
    run(enough, tmp_path)
    assert all(g["rc"] == 1 and not g["kernels"] for g in la.recorded(less, tmp_path)[0])
