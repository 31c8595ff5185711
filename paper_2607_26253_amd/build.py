"""Compile libsara.so (HIP, gfx950) with hipcc and the operators' Python calls
(_operators.so, C++ against torch's headers) with g++, in-tree.  Without torch
only the library is built."""
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libsara.so")
OPERATORS = os.path.join(HERE, "_operators.so")
SOURCES = ["model_kernels.hip", "prefill_kernels.hip", "controller_kernels.hip", "kv8_kernels.hip",
           "score_kernels.hip", "head_kernels.hip", "sara_api.hip"]
FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC",
         # packed fp32 arithmetic is left to no code path (all HIP sources)
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-Wno-unused-result", "-I" + os.path.join(ROOT, "include")]


def hipcc():
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found: the HIP toolchain is required to build libsara")
    return exe


def build(verbose: bool = False) -> str:
    cc = hipcc()
    objdir = os.path.join(HERE, "_build")
    os.makedirs(objdir, exist_ok=True)

    def compile_one(src):
        obj = os.path.join(objdir, src.replace(".hip", ".o"))
        cmd = [cc, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"hipcc failed for {src}:\n{r.stderr}")
        if verbose and r.stderr.strip():
            print(r.stderr)
        return obj

    with ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        objs = list(ex.map(compile_one, SOURCES))
    tmp = OUT + ".tmp"
    r = subprocess.run([cc, "-shared", "-fPIC", "--offload-arch=gfx950", *objs, "-o", tmp],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed:\n{r.stderr}")
    os.replace(tmp, OUT)
    if importlib.util.find_spec("torch"):
        build_operators()
    else:
        print(f"torch is not installed: {os.path.basename(OPERATORS)} (the operators on torch tensors) is not built",
              file=sys.stderr)
    return OUT


def build_operators() -> str:
    """The compiled Python calls; libsara.so is there."""
    import torch

    lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = os.path.join(os.path.dirname(torch.__file__), "include")
    tmp = OPERATORS + ".tmp"
    cmd = [shutil.which("g++") or "c++", "-O2", "-std=c++17", "-fPIC", "-shared",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I" + os.path.join(ROOT, "include"),
           "-I" + include, "-I" + os.path.join(include, "torch", "csrc", "api", "include"),
           "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "operators_binding.cpp"), "-o", tmp, "-L" + HERE, "-L" + lib,
           "-l:libsara.so", "-ltorch_python", "-ltorch_cpu", "-lc10", "-Wl,-rpath,$ORIGIN"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed for operators_binding.cpp:\n{r.stderr}")
    os.replace(tmp, OPERATORS)
    return OPERATORS


if __name__ == "__main__":
    print(build(verbose=True))
