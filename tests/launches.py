"""Records what the sequence calls launch, without a GPU.

A small shared library with the launch functions of the HIP runtime is loaded
before libtq in a child process: the calls run on the host as they are, with
numbers in place of device pointers, and every kernel they would start is
written down with its grid and refused where HIP refuses it.
"""
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_RECORDER = r"""
#include <stddef.h>
#include <stdint.h>
#include <string.h>
typedef struct { uint32_t x, y, z; } dim3;
enum { kKernels = 1 << 14, kLaunches = 1 << 12, kInvalidConfiguration = 9 };
static struct { const void *f; const char *name; } kernels[kKernels];
static int n_kernels, n_launches, error;
static struct { const char *name; dim3 grid, block; } launches[kLaunches];
/* launches nest: a kernel's arguments may launch another */
static struct { dim3 grid, block; size_t shared; void *stream; } stack[8];
static int depth;
void **__hipRegisterFatBinary(const void *d) { static void *h; (void)d; return &h; }
void __hipUnregisterFatBinary(void **m) { (void)m; }
void __hipRegisterVar(void **m, void *v, char *h, char *n, int e, size_t s, int c, int g) {}
void __hipRegisterFunction(void **m, const void *f, char *d, const char *name, unsigned l, void *t, void *b, dim3 *bd,
                           dim3 *gd, int *w)
{
    if (n_kernels < kKernels) kernels[n_kernels].f = f, kernels[n_kernels++].name = name;
}
int __hipPushCallConfiguration(dim3 g, dim3 b, size_t s, void *q)
{
    stack[depth].grid = g, stack[depth].block = b, stack[depth].shared = s, stack[depth++].stream = q;
    return 0;
}
int __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *s, void **q)
{
    depth--;
    *g = stack[depth].grid, *b = stack[depth].block, *s = stack[depth].shared, *q = stack[depth].stream;
    return 0;
}
int hipLaunchKernel(const void *f, dim3 g, dim3 b, void **a, size_t s, void *q)
{
    const char *name = "";
    for (int i = 0; i < n_kernels; i++)
        if (kernels[i].f == f) name = kernels[i].name;
    if (n_launches < kLaunches)
        launches[n_launches].name = name, launches[n_launches].grid = g, launches[n_launches++].block = b;
    /* fewer than 2^32 threads along each axis, at most 65535 workgroups along y and z, none empty */
    if (!g.x || !g.y || !g.z || (uint64_t)g.x * b.x >> 32 || (uint64_t)g.y * b.y >> 32 || g.y > 65535 || g.z > 65535 ||
        (uint64_t)b.x * b.y * b.z > 1024)
        return error = kInvalidConfiguration;
    return 0;
}
int hipGetLastError(void)
{
    const int e = error;
    error = 0;
    return e;
}
int kernel_count(void) { return n_kernels; }
const char *kernel_name(int i) { return kernels[i].name; }
int launch_count(void) { return n_launches; }
void launch_clear(void) { n_launches = 0; }
const char *launch_name(int i) { return launches[i].name; }
uint32_t launch_size(int i, int k)
{
    const dim3 *d = k < 3 ? &launches[i].grid : &launches[i].block;
    return k % 3 == 0 ? d->x : k % 3 == 1 ? d->y : d->z;
}
"""

_CHILD = r"""
import ctypes, json, sys
rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
rec.launch_name.restype = ctypes.c_char_p
rec.launch_size.restype = ctypes.c_uint32
rec.kernel_name.restype = ctypes.c_char_p
lib = ctypes.CDLL(sys.argv[2])
lib.tq_last_error.restype = ctypes.c_char_p
kinds = {"p": ctypes.c_void_p, "i": ctypes.c_int32, "n": ctypes.c_int64, "s": ctypes.c_size_t, "f": ctypes.c_float}
out = []
for name, spec, args in json.load(sys.stdin):
    need = ctypes.c_size_t()
    conv = [ctypes.byref(need) if k == "z" else kinds[k](a) for k, a in zip(spec, args)]
    rec.launch_clear()
    rc = getattr(lib, name)(*conv)
    out.append({"rc": rc, "error": lib.tq_last_error().decode(), "need": need.value,
                "kernels": [[rec.launch_name(i).decode()] + [rec.launch_size(i, k) for k in range(6)]
                            for i in range(rec.launch_count())]})
json.dump({"kernels": [rec.kernel_name(i).decode() for i in range(rec.kernel_count())], "calls": out}, sys.stdout)
"""

P = 1 << 20  # stands for a device pointer, 256-byte aligned

# z: a size_t to be written; p: pointer, i: int32, n: int64, s: size_t, f: float
SPECS = {
    "tq_embed": "pninnpnfpnp",
    "tq_embed_grad_workspace": "nnnz",
    "tq_embed_grad": "pninnpnfpnpsp",
    "tq_gated_scan_workspace": "nnnz",
    "tq_gated_scan": "innnpnnpnnpppnnpppsp",
    "tq_gated_scan_grad": "innnpnnpnnpppnnppnnpnnppsp",
    "tq_layer_norm": "pninnppfpnppp",
    "tq_layer_norm_grad_workspace": "nnz",
    "tq_layer_norm_grad": "pninnppppnpnpppsp",
    "tq_softmax_xent_workspace": "innnz",
    "tq_softmax_xent": "pninnnpnppppsp",
    "tq_softmax_xent_grad_workspace": "innnz",
    "tq_softmax_xent_grad": "pninnnpnpppnpnpppsp",
}
ALL = (1 << 63) - 1  # a workspace of any size


def recorded(calls, tmp_path):
    """[(name, *arguments)] run in a child process: for each {"rc", "error",
    "need", "kernels"}, the last the first 4096 [name, grid x, y, z, workgroup
    x, y, z]; and the names of all kernels there are."""
    so = str(tmp_path / "recorder.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-w", "-x", "c", "-", "-o", so], input=_RECORDER, text=True, check=True)
    asked = [(c[0], SPECS[c[0]], list(c[1:]) + [None] * (len(SPECS[c[0]]) - len(c) + 1)) for c in calls]
    lib = os.environ.get("TQ_LIB_PATH", os.path.join(ROOT, "paper_2003_02989_amd", "libtq.so"))
    r = subprocess.run([sys.executable, "-c", _CHILD, so, lib], input=json.dumps(asked), capture_output=True, text=True,
                       timeout=120)
    assert r.returncode == 0, f"ended with {r.returncode}: {r.stderr[-2000:]}"
    got = json.loads(r.stdout)
    return got["calls"], got["kernels"]


# the calls of the operators on dense arrays; types 0: fp32, 1: bf16, 2: f16

def embed(ty, N, V, D):
    return ("tq_embed", P, D, ty, V, D, P, N, 1.0, P, D, None)


def embed_grad(ty, N, V, D):
    return ("tq_embed_grad", P, D, ty, V, D, P, N, 1.0, P, D, P, ALL, None)


def scan(ty, B, T, D):
    return ("tq_gated_scan", ty, B, T, D, P, T * D, D, P, T * D, D, None, None, P, T * D, D, P, None, P, ALL, None)


def scan_grad(ty, B, T, D):
    return ("tq_gated_scan_grad", ty, B, T, D, P, T * D, D, P, T * D, D, P, None, P, T * D, D, None, P, T * D, D, P,
            T * D, D, P, P, ALL, None)


def norm(ty, N, D):
    return ("tq_layer_norm", P, D, ty, N, D, P, P, 1e-5, P, D, P, P, None)


def norm_grad(ty, N, D):
    return ("tq_layer_norm_grad", P, D, ty, N, D, P, P, P, P, D, P, D, P, P, P, ALL, None)


def xent(ty, N, V, D, ld=0):
    ld = ld or D
    return ("tq_softmax_xent", P, ld, ty, N, V, D, P, ld, P, P, P, P, ALL, None)


def xent_grad(ty, N, V, D, ld=0):
    ld = ld or D
    return ("tq_softmax_xent_grad", P, ld, ty, N, V, D, P, ld, P, P, P, ld, P, ld, P, P, P, ALL, None)
