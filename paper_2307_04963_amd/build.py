"""Build libdycl.so (the C-ABI library with its gfx950 kernels) in-tree, and
_tokens.so, the Python binding of its token operators.

``python -m paper_2307_04963_amd.build`` compiles every source under
``csrc/`` with hipcc for gfx950 and links ``libdycl.so`` next to this file, then
``csrc/binding/`` with the host compiler against torch's headers.
It always recompiles (objects go to ``_build/`` at the repository root).
No GPU is needed: hipcc cross-compiles.  The library itself needs hipcc alone:
where torch, its or Python's headers or the host compiler are missing, the
binding is left out (importing ``experts`` says so) and the rest is built.
"""

from __future__ import annotations

import concurrent.futures as cf
import glob
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libdycl.so")
BINDING = os.path.join(PKG, "_tokens.so")
BUILD = os.path.join(ROOT, "_build")
ARCH = "gfx950"

# -packed-fp32-ops off: the compiler must not form v_pk_{add,mul,fma}_f32
HIPCC_FLAGS = ["-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-Wall", "-Wno-unused-result",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def hipcc() -> str:
    for cand in (os.environ.get("HIPCC"), "/opt/rocm/bin/hipcc", shutil.which("hipcc")):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("hipcc not found (ROCm is required to build libdycl.so)")


def _compile(src: str) -> str:
    obj = os.path.join(BUILD, os.path.basename(src) + ".o")
    cmd = [hipcc()] + HIPCC_FLAGS + ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _cxx() -> str:
    return os.environ.get("CXX", "g++")


def _binding_lacks() -> str:
    """What the binding cannot be built without and is not here, or ""."""
    if not shutil.which(_cxx()):
        return f"the host compiler {_cxx()}"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    try:
        from torch.utils import cpp_extension
    except ImportError:
        return "torch"
    if not any(os.path.exists(os.path.join(d, "ATen", "ATen.h")) for d in cpp_extension.include_paths()):
        return "torch's C++ headers"
    return ""


def _compile_binding() -> str:
    """The binding's object: host code that sees torch's and HIP's headers."""
    import torch
    from torch.utils import cpp_extension
    src = os.path.join(CSRC, "binding", "tokens.cpp")
    obj = os.path.join(BUILD, "binding_tokens.o")
    rocm = os.path.dirname(os.path.dirname(hipcc()))
    cmd = [_cxx(), "-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-isystem", sysconfig.get_paths()["include"],
           "-isystem", os.path.join(rocm, "include")]
    for inc in cpp_extension.include_paths():
        cmd += ["-isystem", inc]
    cmd += ["-c", src, "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return obj


def _link_binding(obj: str) -> None:
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")
    tmp = BINDING + ".tmp"
    # (torch's libraries are in the process already; the library beside it is found by its own folder)
    cmd = [_cxx(), "-shared", "-fPIC", "-o", tmp, obj, "-L" + PKG, "-l:libdycl.so", "-L" + libs, "-lc10", "-lc10_hip",
           "-ltorch_cpu", "-ltorch_hip", "-ltorch_python", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, BINDING)


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.cpp")) + glob.glob(os.path.join(CSRC, "*.hip")))
    workers = min(len(srcs), max(1, min(16, os.cpu_count() or 1)))
    lacks = _binding_lacks()
    with cf.ThreadPoolExecutor(workers) as ex:
        binding = None if lacks else ex.submit(_compile_binding)
        objs = list(ex.map(_compile, srcs))
    tmp = OUT + ".tmp"
    cmd = [hipcc(), "-shared", "-fPIC", f"--offload-arch={ARCH}", "-o", tmp] + objs
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    # every symbol of the library's own namespace must be defined (a kernel
    # template whose host-side stub was not emitted links fine and fails at load)
    nm = subprocess.run(["nm", "-u", "-C", tmp], capture_output=True, text=True)
    missing = [ln.strip() for ln in nm.stdout.splitlines() if "dycl::" in ln]
    if missing:
        os.remove(tmp)
        raise RuntimeError("undefined symbols in the library:\n" + "\n".join(missing[:20]))
    os.replace(tmp, OUT)
    if binding is None:
        if os.path.exists(BINDING):
            os.remove(BINDING)             # (of another library)
        print(f"built {OUT}; without {lacks} the token operators' Python binding is left out", file=sys.stderr, flush=True)
        return OUT
    _link_binding(binding.result())
    if verbose:
        print("built", OUT, "and", BINDING, flush=True)
    return OUT


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
