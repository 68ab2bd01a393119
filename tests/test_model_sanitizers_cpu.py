"""AddressSanitizer + UndefinedBehaviorSanitizer run of the host half of the
operators of selective models (model_abi.cpp, with the error handling of
tq_abi.cpp): the refusal tests against a library whose host code is sanitized.
The launchers in the kernel sources are linked as built."""
import os
import subprocess

import pytest

from test_sanitizers_cpu import CLANGXX, HIPCC, PKG, ROOT, _clang_runtime, _run_tests


def test_model_abi_under_asan_ubsan(tmp_path):
    rt = _clang_runtime()
    built = [os.path.join(PKG, "_build", n + ".o") for n in
             ("kernels.hip", "seq_embed.hip", "seq_scan.hip", "seq_norm.hip", "seq_xent.hip", "model_scan.hip",
              "model_conv.hip", "model_clip.hip", "model_beam.hip")]
    if rt is None or not os.path.exists(CLANGXX):
        pytest.skip("the ROCm clang ASan runtime is not installed")
    if not all(os.path.exists(o) for o in built):
        pytest.skip("libtq is not built (python -m paper_2003_02989_amd.build)")
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-fno-omit-frame-pointer",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-Xarch_host", "-fno-sanitize-recover=undefined",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-I", os.path.join(ROOT, "include"), "-I", os.path.join(PKG, "_build")]
    procs, objs = [], []
    for src in ("program.cpp", "tq_abi.cpp", "jit.cpp", "seq_abi.cpp", "model_abi.cpp"):
        obj = str(tmp_path / (src + ".o"))
        objs.append(obj)
        procs.append(subprocess.Popen([HIPCC] + flags + ["-c", os.path.join(PKG, "csrc", src), "-o", obj],
                                      stdout=subprocess.PIPE, stderr=subprocess.STDOUT))
    for p in procs:
        out = p.communicate()[0]
        assert p.returncode == 0, out.decode()[-3000:]
    lib = str(tmp_path / "libtq_san.so")
    subprocess.check_call([CLANGXX, "-shared", "-fPIC", "-fsanitize=address,undefined", "-shared-libasan", "-o", lib]
                          + objs + built + ["-L/opt/rocm/lib", "-lamdhip64", "-lhiprtc", "-pthread",
                                            "-Wl,--no-undefined", "-Wl,-rpath,/opt/rocm/lib"])
    _run_tests(["test_model_abi_cpu.py"], {"TQ_LIB_PATH": lib}, rt)
