"""Build ``libleapfrog.so`` in-tree with nvcc for sm_100a, and ``_marshal.so`` with g++ (tensor marshalling
of the layer operators, against the installed torch's headers; without torch it is left out and the C library alone is built).

Run as ``python -m paper_1801_04928_b200.build`` or call :func:`build`.  The shared library
lands beside this file; nothing is installed elsewhere and nothing is compiled at import time.
"""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
OBJ = os.path.join(PKG, "_build")
LIB = os.path.join(PKG, "libleapfrog.so")

SOURCES = ["lf_api.cu", "lf_kernels_b1.cu", "lf_kernels_batch.cu", "lf_persistent.cu", "lf_columns.cu",
           "lf_gemm_tf32.cu", "lf_delta_gemm_tc.cu", "lf_ops_api.cu", "lf_rows.cu", "lf_linear_tc.cu",
           "lf_linear_stream.cu", "lf_layer_norm.cu", "lf_blocks_tc.cu", "lf_blocks_stream.cu", "lf_distill.cu"]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC", "-Xptxas", "-v", "-I", INCLUDE, "-I", CSRC]


MARSHAL_SRC = os.path.join(CSRC, "lf_marshal.cpp")
MARSHAL = os.path.join(PKG, "_marshal.so")


def _build_marshal(force: bool) -> None:
    spec = importlib.util.find_spec("torch")
    if spec is None or spec.origin is None:
        sys.stderr.write("torch not found: _marshal.so, the layer operators on torch tensors, is not built\n")
        return
    torch_dir = os.path.dirname(spec.origin)
    # the module fits the torch and the Python it was built against: others make it stale
    version = os.path.join(torch_dir, "version.py")
    against = f"{sys.version}\n{torch_dir}\n" + (open(version).read() if os.path.exists(version) else "")
    stamp = os.path.join(OBJ, os.path.basename(MARSHAL) + ".torch")
    same = os.path.exists(stamp) and open(stamp).read() == against
    if not force and same and not _stale(MARSHAL, [MARSHAL_SRC, os.path.join(INCLUDE, "leapfrog.h")]):
        return
    inc = os.path.join(torch_dir, "include")
    tmp = MARSHAL + f".tmp{os.getpid()}"
    # no run path: torch is loaded before the module, which finds its libraries by name
    r = subprocess.run(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-w", MARSHAL_SRC, "-o", tmp, "-I", INCLUDE,
                        "-I", sysconfig.get_paths()["include"], "-I", inc, "-I", os.path.join(inc, "torch", "csrc", "api", "include"),
                        "-I", os.path.join(os.path.dirname(os.path.dirname(_nvcc())), "include"),
                        "-L", os.path.join(torch_dir, "lib"), "-ltorch_python", "-ltorch_cpu", "-ltorch", "-lc10"],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"g++ failed on lf_marshal.cpp:\n{r.stdout}\n{r.stderr}")
    os.replace(tmp, MARSHAL)
    with open(stamp, "w") as f:
        f.write(against)


def _nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the CUDA library cannot be built")
    return exe


def _stale(target: str, deps: list[str]) -> bool:
    if not os.path.exists(target):
        return True
    t = os.path.getmtime(target)
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile every translation unit and link the shared library.  Returns its path."""
    os.makedirs(OBJ, exist_ok=True)
    headers = [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".h", ".cuh"))]
    headers.append(os.path.join(INCLUDE, "leapfrog.h"))
    nvcc = _nvcc()

    def compile_one(src: str) -> str:
        path = os.path.join(CSRC, src)
        obj = os.path.join(OBJ, src.replace(".cu", ".o"))
        if force or _stale(obj, [path] + headers):
            r = subprocess.run([nvcc, *NVCC_FLAGS, "-c", path, "-o", obj],
                               capture_output=True, text=True)
            with open(obj + ".log", "w") as f:
                f.write(r.stdout + r.stderr)
            if r.returncode != 0:
                raise RuntimeError(f"nvcc failed on {src}:\n{r.stdout}\n{r.stderr}")
            if verbose:
                sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        marshal = ex.submit(_build_marshal, force)
        objs = list(ex.map(compile_one, SOURCES))
    if force or _stale(LIB, objs):
        tmp = LIB + f".tmp{os.getpid()}"
        r = subprocess.run([nvcc, "-shared", "-o", tmp, *objs, "-gencode",
                            "arch=compute_100a,code=sm_100a"], capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"link failed:\n{r.stdout}\n{r.stderr}")
        os.replace(tmp, LIB)
    marshal.result()                 # (last: what goes wrong there does not keep the library from being linked)
    return LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose=True))
