"""Builds libsprinter.so (HIP kernels + C ABI) in-tree for gfx950 with hipcc."""
from __future__ import annotations
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libsprinter.so")
TENSORS = os.path.join(PKG, "_tensors.so")
NATIVE_BENCH = os.path.join(PKG, "native_bench")
SOURCES = ["k_norm.hip", "k_gemm.hip", "k_gemm_norm.hip", "k_gemm_tile.hip", "k_attn.hip", "k_lmhead.hip", "k_control.hip", "k_sd.hip", "k_route.hip", "k_experts.hip", "k_experts_tile.hip",
           "k_block_norm.hip", "k_cache.hip", "k_tree_attn.hip", "k_logits.hip", "ops.cpp", "abi.cpp"]
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
         # packed-fp32 VALU forms are kept off on the test machines
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         # the first argument words of a kernel are loaded into registers with its dispatch
         "-mllvm", "-amdgpu-kernarg-preload-count=14",
         "-Wno-unused-command-line-argument"]


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops' is not a recognized feature" not in l)
    if out.strip() and verbose:
        print(out, flush=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed:\n" + out)


def tensors_lack() -> str:
    """What the extension of the torch entry points needs and is not here; callers of the C library need hipcc alone."""
    import sysconfig
    if shutil.which("g++") is None:
        return "g++"
    try:
        from torch.utils import cpp_extension
    except ImportError:
        return "torch"
    for where, name in (([sysconfig.get_paths()["include"]], "Python.h"), (cpp_extension.include_paths(), os.path.join("torch", "extension.h"))):
        if not any(os.path.exists(os.path.join(p, name)) for p in where):
            return name
    return ""


def build_tensors(verbose: bool = True) -> None:
    """The Python extension that looks tensors over for the operators (csrc/tensors.cpp; host code only)."""
    import sysconfig
    from torch.utils import cpp_extension
    import torch
    _run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
          *("-isystem" + p for p in cpp_extension.include_paths()), "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "tensors.cpp"), "-o", TENSORS,
          *("-L" + p for p in cpp_extension.library_paths()), "-ltorch_python", "-ltorch_cpu", "-lc10"], verbose)


def build_library(verbose: bool = True) -> str:
    """Every source is compiled (in parallel) on each call, then linked into the shared library.  The extension is left out, with a word, where what it needs is not here."""
    from concurrent.futures import ThreadPoolExecutor
    lack = tensors_lack()
    if lack:
        print(f"no {lack}: _tensors.so, which the cache in pages and the adjustments of logits need on torch tensors, is not built", flush=True)
        if os.path.exists(TENSORS):
            os.remove(TENSORS)                           # (of other sources)
    objdir = os.path.join(PKG, "_build")
    os.makedirs(objdir, exist_ok=True)
    objs = [os.path.join(objdir, s + ".o") for s in SOURCES]
    cmds = [["hipcc", *FLAGS, "-x", "hip", "-c", os.path.join(CSRC, s), "-o", o] for s, o in zip(SOURCES, objs)]
    with ThreadPoolExecutor(max_workers=len(cmds) + 1) as ex:
        tensors = None if lack else ex.submit(build_tensors, verbose)
        list(ex.map(lambda c: _run(c, verbose), cmds))
        if tensors:
            tensors.result()
    _run(["hipcc", "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", LIB], verbose)
    # the Python-free runner of dumped workloads (hardware-counter runs); it only uses the public C ABI
    _run(["hipcc", *FLAGS, "-x", "hip", os.path.join(CSRC, "native_bench.cpp"), "-L" + PKG, "-lsprinter",
          "-Wl,-rpath,$ORIGIN", "-o", NATIVE_BENCH], verbose)
    return LIB


if __name__ == "__main__":
    build_library()
    print("built", LIB)
    sys.exit(0)
