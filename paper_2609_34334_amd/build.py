"""Builds libhoccl.so in-tree with hipcc for gfx950, and the extension module
_tensors.so, which reads lists of torch tensors, with the host compiler.

Every source is compiled to an object in parallel, then linked into
``paper_2609_34334_amd/libhoccl.so`` next to this file.  Always rebuilds.
"""
import os
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
BUILD = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libhoccl.so")
TENSORS = os.path.join(HERE, "_tensors.so")
SOURCES = ["api.cpp", "plan.cpp", "proxy.cpp", "schedule.cpp", "kernels.hip", "handshake.hip",
           "scratch.hip", "ceilings.hip", "ipc.cpp", "mailbox.cpp", "shard_ops.cpp", "adamw.hip",
           "rmsnorm.hip", "balance.hip"]
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# The packed-fp32 feature is switched off for device code: the library
# writes plain scalar float arithmetic and never wants v_pk_*_f32.
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops"]


def _compile(src):
    obj = os.path.join(BUILD, os.path.splitext(src)[0] + ".o")
    cmd = [HIPCC] + FLAGS + ["-c", os.path.join(CSRC, src), "-o", obj]
    r = subprocess.run(cmd, capture_output=True, text=True)
    out = "\n".join(l for l in (r.stdout + r.stderr).splitlines()
                    if "packed-fp32-ops" not in l)
    if r.returncode != 0:
        raise RuntimeError(f"compiling {src} failed:\n{out}")
    return obj


def _tensors():
    import torch
    home = os.path.dirname(torch.__file__)
    tmp = TENSORS + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-isystem", os.path.join(home, "include"),
           "-isystem", os.path.join(home, "include", "torch", "csrc", "api", "include"),
           "-I" + sysconfig.get_paths()["include"], os.path.join(CSRC, "tensors.cpp"), "-o", tmp,
           "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"building _tensors.so failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, TENSORS)


def build(verbose=True):
    os.makedirs(BUILD, exist_ok=True)
    with ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as ex:
        tensors = ex.submit(_tensors)
        objs = list(ex.map(_compile, SOURCES))
        tensors.result()
    tmp = LIB + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp] + objs + [
        "-L/opt/rocm/lib", "-lhsa-runtime64", "-lamdhip64", "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"linking libhoccl.so failed:\n{r.stdout}{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}", file=sys.stderr)
    return LIB


if __name__ == "__main__":
    build()
