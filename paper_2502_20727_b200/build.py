"""Build the CUDA library in-tree with nvcc for sm_100a (cross-compiles without a GPU)."""
from __future__ import annotations

import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libspd_b200.so")
CALLS = os.path.join(HERE, "_calls.so")  # Python module over the library (csrc/binding.cpp)
NVCC = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC",
         "--expt-relaxed-constexpr"]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith(".cu"))


def _deps():
    out = sources() + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h", ".cpp"))]
    out.append(os.path.join(os.path.dirname(HERE), "include", "spd.h"))
    return out


def build(force: bool = False, verbose: bool = False, trace: bool = False) -> str:
    """trace=True builds libspd_b200_trace.so with the in-kernel timeline compiled in (-DSPD_TRACE)."""
    lib = LIB.replace(".so", "_trace.so") if trace else LIB
    newest = max(os.path.getmtime(p) for p in _deps())
    made = [lib] if trace else [lib, CALLS]
    if not force and all(os.path.exists(f) and os.path.getmtime(f) >= newest for f in made):
        return lib
    objdir = os.path.join(HERE, "_build", "trace" if trace else "plain")
    os.makedirs(objdir, exist_ok=True)
    objs = []
    procs = []
    binding = os.path.join(objdir, "binding.o")
    if not trace:
        torch_dir = os.path.dirname(importlib.util.find_spec("torch").origin)
        cmd = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-c", os.path.join(CSRC, "binding.cpp"), "-o", binding,
               f"-I{torch_dir}/include", f"-I{torch_dir}/include/torch/csrc/api/include", f"-I{sysconfig.get_paths()['include']}", "-I/usr/local/cuda/include"]
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for src in sources():
        obj = os.path.join(objdir, os.path.basename(src)[:-3] + ".o")
        objs.append(obj)
        cmd = [NVCC, *FLAGS, "-c", src, "-o", obj] + (["-Xptxas", "-v"] if verbose else []) + \
              (["-DSPD_TRACE", "-rdc=true"] if trace else [])
        procs.append((cmd, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for cmd, pr in procs:
        out, _ = pr.communicate()
        if verbose or pr.returncode:
            sys.stderr.write(out)
        if pr.returncode:
            raise RuntimeError("nvcc failed: " + " ".join(cmd))
    cmd = [NVCC, "-shared", "-o", lib, *objs, "-gencode", "arch=compute_100a,code=sm_100a"]
    subprocess.run(cmd, check=True)
    if not trace:
        libs = [f"-L{torch_dir}/lib", "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
        subprocess.run(["g++", "-shared", "-o", CALLS, binding, f"-L{HERE}", "-l:" + os.path.basename(LIB), *libs, "-Wl,-rpath,$ORIGIN"], check=True)
    return lib


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv, trace="--trace" in sys.argv))
