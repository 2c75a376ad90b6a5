"""Build the CUDA library libqwm.so in-tree for sm_103a.

Each .cu translation unit is compiled by its own nvcc process (in parallel),
then linked into ``paper_2609_26425_gb300/_build/libqwm.so`` with the static
CUDA runtime, so the library loads without a GPU and without libcudart.so.
"""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "_build")
LIB = os.path.join(OUT, "libqwm.so")
BINDING = os.path.join(OUT, "qwm_binding.so")  # csrc/binding.cpp, against PyTorch's headers
STAMP = os.path.join(OUT, "qwm_binding.txt")   # which PyTorch that was
SOURCES = ["qwm_api.cu", "append.cu", "append_fused.cu", "append_fused_r8.cu", "append_fused_r16.cu",
           "append_fused_r32.cu", "append_generic.cu", "append_full.cu", "attend.cu", "fit.cu", "qstats.cu",
           "metrics.cu", "rope.cu", "paged_api.cu", "paged_step.cu", "paged_chunk.cu"]
ARCH = ["-gencode", "arch=compute_103a,code=sm_103a"]
FLAGS = ["-O3", "-lineinfo", "-std=c++17", "-Xcompiler", "-fPIC", "-Xcompiler", "-fvisibility=hidden",
         "--expt-relaxed-constexpr"]


def nvcc() -> str:
    p = shutil.which("nvcc")
    if p:
        return p
    p = "/usr/local/cuda/bin/nvcc"
    if os.path.exists(p):
        return p
    raise RuntimeError("nvcc not found: the CUDA toolkit is required to build libqwm.so")


def _deps():
    files = [os.path.join(CSRC, f) for f in os.listdir(CSRC)]
    files.append(os.path.join(HERE, "..", "include", "qwm.h"))
    return files


def _built_with() -> str:
    """The PyTorch and the Python that the binding is compiled against."""
    import torch
    return "\n".join((torch.__version__, os.path.dirname(torch.__file__), str(torch._C._GLIBCXX_USE_CXX11_ABI),
                      sys.version, sysconfig.get_paths()["include"]))


def up_to_date() -> bool:
    if not os.path.exists(LIB) or not os.path.exists(BINDING):
        return False
    try:
        with open(STAMP) as f:
            if f.read() != _built_with():
                return False
    except FileNotFoundError:
        return False
    t = min(os.path.getmtime(LIB), os.path.getmtime(BINDING))
    return all(os.path.getmtime(f) <= t for f in _deps())


def build(force: bool = False, verbose: bool = False, ptxas_info: bool = False) -> str:
    if not force and up_to_date():
        return LIB
    os.makedirs(OUT, exist_ok=True)
    cc = nvcc()
    extra = ["-Xptxas", "-v"] if ptxas_info else []

    def compile_one(src):
        obj = os.path.join(OUT, src.replace(".cu", ".o"))
        cmd = [cc, *ARCH, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"nvcc failed for {src}:\n{r.stderr}")
        if verbose or ptxas_info:
            sys.stderr.write(r.stderr)
        return obj

    def compile_binding():
        import torch  # headers and library paths only
        inc = [os.path.join(os.path.dirname(torch.__file__), "include"), sysconfig.get_paths()["include"],
               os.path.join(os.path.dirname(os.path.realpath(cc)), "..", "include")]
        obj = os.path.join(OUT, "binding.o")
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden",
               f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", *("-I" + i for i in inc), "-c",
               os.path.join(CSRC, "binding.cpp"), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"g++ failed for binding.cpp:\n{r.stderr}")
        return obj, os.path.join(os.path.dirname(torch.__file__), "lib")

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        bound = ex.submit(compile_binding)
        objs = list(ex.map(compile_one, SOURCES))
        bobj, torch_lib = bound.result()
    tmp = LIB + f".tmp{os.getpid()}"
    cmd = [cc, *ARCH, "-shared", "--cudart", "static", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, LIB)
    tmp = BINDING + f".tmp{os.getpid()}"
    cmd = ["g++", "-shared", "-o", tmp, bobj, "-L" + OUT, "-lqwm", "-Wl,-rpath,$ORIGIN", "-L" + torch_lib,
           "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda", "-Wl,-rpath," + torch_lib]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, BINDING)
    with open(STAMP, "w") as f:
        f.write(_built_with())
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True, ptxas_info="--ptxas" in sys.argv))
