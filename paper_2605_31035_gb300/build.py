"""Build libmixfp4.so (sm_103a) in-tree with nvcc, and the Python binding
_binding.so of its latency-bound entry points with the host compiler.

Each translation unit under csrc/ is compiled in parallel with
``-gencode arch=compute_103a,code=sm_103a -lineinfo`` and linked into a
shared library with the CUDA runtime linked statically, so the library loads
next to any PyTorch build.  Objects go to ``_build/`` (git-ignored).
"""
from __future__ import annotations

import concurrent.futures as cf
import os
import shutil
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmixfp4.so")
BINDING = os.path.join(HERE, "_binding.so")
BINDING_ABI = os.path.join(HERE, "_binding.abi")  # what _binding.so was compiled for
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

SOURCES = ["api.cu", "quantize.cu", "train.cu", "gemm.cu", "gemm_f16a.cu", "fewrows.cu", "native.cu", "candidates.cu", "noalloc.cu", "selftest.cu",
           "kvcache.cu", "kvmove.cu", "attention.cu", "tree_attention.cu", "lora.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
NVCC_FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas", "-v",
              "--ftz=false", "--prec-div=true", "--prec-sqrt=true", "--fmad=false",
              f"-I{INCLUDE}"]


def _nvcc() -> str:
    for cand in (shutil.which("nvcc"), "/usr/local/cuda/bin/nvcc"):
        if cand and os.path.exists(cand):
            return cand
    raise RuntimeError("nvcc not found: the MixFP4 CUDA library cannot be built")


def _deps():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    files.append(os.path.join(INCLUDE, "mixfp4.h"))
    return files


def abi() -> str:
    """The Python and the torch that a compiled binding belongs to."""
    import torch
    return f"{sysconfig.get_config_var('SOABI')} torch {torch.__version__} cxx11 {int(torch._C._GLIBCXX_USE_CXX11_ABI)}\n"


def binding_fits() -> bool:
    """Whether _binding.so was compiled for this Python and this torch: one for others may fail to load, or read tensors by
    another layout."""
    try:
        with open(BINDING_ABI) as f:
            return f.read() == abi()
    except OSError:
        return False


def up_to_date() -> bool:
    if not (os.path.exists(LIB) and os.path.exists(BINDING) and binding_fits()):
        return False
    t = min(os.path.getmtime(LIB), os.path.getmtime(BINDING))
    return all(os.path.getmtime(f) <= t for f in _deps())


def _compile(src: str) -> tuple[str, str]:
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [_nvcc(), *ARCH, *NVCC_FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"nvcc failed for {src}:\n{res.stderr}")
    return obj, res.stderr


def _compile_binding() -> str:
    """csrc/binding.cpp against this interpreter's and this torch's headers."""
    import torch
    root = os.path.dirname(torch.__file__)
    obj = os.path.join(BUILD, "binding.o")
    cmd = [shutil.which("g++") or shutil.which("c++") or "g++", "-O2", "-std=c++17", "-fPIC",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", f"-I{INCLUDE}",
           f"-I{sysconfig.get_paths()['include']}", f"-I{root}/include", f"-I{root}/include/torch/csrc/api/include",
           "-c", os.path.join(CSRC, "binding.cpp"), "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"the host compiler failed for binding.cpp:\n{res.stderr}")
    return obj


def _link_binding(obj: str):
    import torch
    tmp = BINDING + f".tmp{os.getpid()}"
    cmd = [shutil.which("g++") or shutil.which("c++") or "g++", "-shared", "-o", tmp, obj, f"-L{HERE}",
           f"-l:{os.path.basename(LIB)}", "-Wl,-rpath,$ORIGIN",
           f"-L{os.path.dirname(torch.__file__)}/lib", "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link of the binding failed:\n{res.stderr}")
    if os.path.exists(BINDING_ABI):
        os.remove(BINDING_ABI)  # never one module's beside another
    os.replace(tmp, BINDING)
    with open(BINDING_ABI + f".tmp{os.getpid()}", "w") as f:
        f.write(abi())
    os.replace(f.name, BINDING_ABI)


def build(force: bool = False, verbose: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(BUILD, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        binding = ex.submit(_compile_binding)
        results = list(ex.map(_compile, SOURCES))
        binding = binding.result()
    if verbose:
        for _, log in results:
            sys.stderr.write(log)
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [_nvcc(), *ARCH, "-shared", "-cudart", "static", "-o", tmp] + [o for o, _ in results]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stderr}")
    os.replace(tmp, LIB)
    _link_binding(binding)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
