"""Builds libgsa_b200.so (the C-ABI library) in-tree with nvcc for sm_100a, and the small extension that calls it from Python."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
LIB_PATH = os.path.join(_PKG, "libgsa_b200.so")
CALL_PATH = os.path.join(_PKG, "_gsa_call" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
CXX = os.environ.get("CXX", "g++")

FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-I", os.path.join(_ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _stale() -> bool:
    if not os.path.exists(LIB_PATH) or not os.path.exists(CALL_PATH):
        return True
    t = min(os.path.getmtime(LIB_PATH), os.path.getmtime(CALL_PATH))
    deps = sources() + [os.path.join(CSRC, "gsa_call.cpp")] + glob.glob(os.path.join(CSRC, "*.cuh")) + glob.glob(os.path.join(_ROOT, "include", "*.h"))
    return any(os.path.getmtime(d) > t for d in deps)


def _call_command(out: str) -> list:
    """Compiles the extension against the installed PyTorch, whose libraries are loaded by the time it is."""
    t = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")
    inc = [sysconfig.get_paths()["include"], os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"), cuda,
           os.path.join(_ROOT, "include")]
    return [CXX, "-O2", "-std=c++17", "-shared", "-fPIC", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            *[x for i in inc for x in ("-I", i)], os.path.join(CSRC, "gsa_call.cpp"), "-o", out,
            "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ and link the shared library.  No GPU needed."""
    if not force and not _stale():
        return LIB_PATH
    objdir = os.path.join(_PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, procs = [], []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [NVCC, *FLAGS, "-c", src, "-o", obj] + (["-Xptxas", "-v"] if verbose else [])
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    call = CALL_PATH + f".tmp{os.getpid()}"
    cmd = _call_command(call)
    procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode:
            sys.stderr.write(out)
        if pr.returncode:
            raise RuntimeError("failed: " + " ".join(cmd))
    tmp = LIB_PATH + f".tmp{os.getpid()}"
    subprocess.check_call([NVCC, "-shared", "-o", tmp, *objs, "-lcudart", "-ldl"])
    os.replace(tmp, LIB_PATH)
    os.replace(call, CALL_PATH)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
