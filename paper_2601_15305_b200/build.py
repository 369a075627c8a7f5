"""Builds libgsa_b200.so (the C-ABI library) in-tree with nvcc for sm_100a, and the small extension that calls it from Python."""
from __future__ import annotations

import glob
import os
import subprocess
import sys
import sysconfig
import warnings

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_PKG)
CSRC = os.path.join(_PKG, "csrc")
LIB_PATH = os.path.join(_PKG, "libgsa_b200.so")
CALL_PATH = os.path.join(_PKG, "_gsa_call" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
CALL_STAMP = os.path.join(_PKG, "_build", "_gsa_call.built_for")
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
CXX = os.environ.get("CXX", "g++")

FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
         "--expt-relaxed-constexpr", "-Xcompiler", "-fPIC", "-I", os.path.join(_ROOT, "include"), "-I", CSRC]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.cu")))


def _older(out: str, deps: list) -> bool:
    return not os.path.exists(out) or any(os.path.getmtime(d) > os.path.getmtime(out) for d in deps)


def _headers() -> list:
    return glob.glob(os.path.join(_ROOT, "include", "*.h"))


def built_for() -> str:
    """What the extension is compiled against: it holds inlined parts of PyTorch and of the interpreter."""
    return f"PyTorch {torch.__version__}, C++ ABI {int(torch.compiled_with_cxx11_abi())}, {sysconfig.get_config_var('SOABI')}"


def _library_stale() -> bool:
    return _older(LIB_PATH, sources() + glob.glob(os.path.join(CSRC, "*.cuh")) + _headers())


def _call_stale() -> bool:
    if _older(CALL_PATH, [os.path.join(CSRC, "gsa_call.cpp")] + _headers()) or not os.path.exists(CALL_STAMP):
        return True
    with open(CALL_STAMP) as f:
        return f.read() != built_for()


def _stale() -> bool:
    return _library_stale() or _call_stale()


def _call_command(out: str) -> list:
    """Compiles the extension against the installed PyTorch, whose libraries are loaded by the time it is."""
    t = os.path.dirname(torch.__file__)
    cuda = os.path.join(os.path.dirname(os.path.dirname(NVCC)), "include")
    inc = [sysconfig.get_paths()["include"], os.path.join(t, "include"), os.path.join(t, "include", "torch", "csrc", "api", "include"), cuda,
           os.path.join(_ROOT, "include")]
    return [CXX, "-O2", "-std=c++17", "-shared", "-fPIC", "-w", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
            f'-DGSA_BUILT_FOR="{built_for()}"',
            *[x for i in inc for x in ("-I", i)], os.path.join(CSRC, "gsa_call.cpp"), "-o", out,
            "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10", "-lc10_cuda"]


def _finish(cmd: list, pr, verbose: bool) -> None:
    out, _ = pr.communicate()
    if verbose or pr.returncode:
        sys.stderr.write(out)
    if pr.returncode:
        raise RuntimeError("failed: " + " ".join(cmd))


def _start(cmd: list):
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _build_library(verbose: bool) -> None:
    objdir = os.path.join(_PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs, procs = [], []
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [NVCC, *FLAGS, "-c", src, "-o", obj] + (["-Xptxas", "-v"] if verbose else [])
        procs.append((cmd, _start(cmd)))
    for cmd, pr in procs:
        _finish(cmd, pr, verbose)
    tmp = os.path.join(objdir, f"library.{os.getpid()}.so")
    subprocess.check_call([NVCC, "-shared", "-o", tmp, *objs, "-lcudart", "-ldl"])
    os.replace(tmp, LIB_PATH)


def _build_call(verbose: bool) -> None:
    """One that was built for something else goes first: what is left by a failure is no extension rather than that one."""
    for old in (CALL_STAMP, CALL_PATH):
        if os.path.exists(old):
            os.remove(old)
    os.makedirs(os.path.dirname(CALL_STAMP), exist_ok=True)
    tmp = os.path.join(os.path.dirname(CALL_STAMP), f"call.{os.getpid()}.so")
    cmd = _call_command(tmp)
    _finish(cmd, _start(cmd), verbose)
    os.replace(tmp, CALL_PATH)
    with open(CALL_STAMP, "w") as f:
        f.write(built_for())


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every .cu under csrc/ and link the shared library, then the extension.  No GPU needed.

    The library needs nvcc alone.  The extension also needs a C++ compiler and the headers of Python and PyTorch: where it cannot be
    built the library stands, a warning says why, and the cache's calls from Python, which alone go through it, raise.
    """
    if force or _library_stale():
        _build_library(verbose)
    if force or _call_stale():
        try:
            _build_call(verbose)
        except (OSError, RuntimeError) as e:
            warnings.warn(f"the extension of the cache's calls was not built ({e}); everything else was", RuntimeWarning, stacklevel=2)
    return LIB_PATH


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
