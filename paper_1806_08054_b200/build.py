"""Build the CUDA library in-tree for sm_100a (no GPU needed: nvcc cross-compiles)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB = os.path.join(_HERE, "libecq.so")
SOURCES = ["ecq_api.cu", "ecq_token.cu", "ecq_muon.cu", "ecq_act8.cu", "ecq_product8.cu"]
HEADERS = ["ecq_common.cuh", "ecq_encode.cuh", "ecq_decode.cuh", "ecq_decode_ring.cuh", "ecq_stats.cuh", "ecq_entropy.cuh",
           "ecq_host.h", "ecq_elem.cuh", "ecq_token.cuh", "ecq_tensor.cuh", "ecq_muon.cuh",
           "ecq_act8.cuh", "ecq_act8_kernels.cuh", "ecq_act8_host.h", "ecq_ring.h",
           "ecq_product8.cuh"]

NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    # every fp32 operation of the codec is an explicit round-to-nearest intrinsic;
    # contraction is also switched off globally so nothing can be fused behind them
    "-fmad=false", "-shared", "-Xcompiler", "-fPIC", "--threads", "0",
]


def _stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = [os.path.join(CSRC, f) for f in SOURCES + HEADERS]
    deps.append(os.path.join(os.path.dirname(_HERE), "include", "ecq.h"))
    return any(os.path.getmtime(p) > t for p in deps)


MARSHAL = os.path.join(_HERE, "_marshal.so")


def build_marshal(force: bool = False) -> bool:
    """Compile the binding's argument marshalling (``csrc/ecq_marshal.cpp``) next to this file.  Where that cannot
    be done (no headers of Python or torch) the binding does the same in Python, a few microseconds a call slower."""
    source = os.path.join(CSRC, "ecq_marshal.cpp")
    if not force and os.path.exists(MARSHAL) and os.path.getmtime(MARSHAL) >= os.path.getmtime(source):
        return True
    import sysconfig
    import torch
    libs = os.path.join(os.path.dirname(torch.__file__), "lib")      # loaded by torch before this is
    base = os.path.join(os.path.dirname(torch.__file__), "include")
    tmp = MARSHAL + ".tmp.%d" % os.getpid()
    cmd = [os.environ.get("CXX", "g++"), "-std=c++17", "-O2", "-fPIC", "-shared", "-I" + sysconfig.get_paths()["include"], "-I" + base,
           "-I" + os.path.join(base, "torch", "csrc", "api", "include"), source, "-o", tmp,
           "-L" + libs, "-ltorch_python", "-ltorch_cpu", "-lc10"]
    try:
        done = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        print("ecq_marshal.cpp is not built: %s" % e)
        return False
    if done.returncode:
        print("ecq_marshal.cpp is not built:\n" + done.stderr[-2000:])
        return False
    os.replace(tmp, MARSHAL)
    return True


def build_library(force: bool = False, verbose: bool = False) -> str:
    """Compile ``libecq.so`` next to this file if it is missing or out of date."""
    build_marshal(force)
    if force or _stale():
        nvcc = os.environ.get("NVCC", "nvcc")
        tmp = LIB + ".tmp.%d" % os.getpid()
        cmd = [nvcc] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
              ["-o", tmp] + [os.path.join(CSRC, s) for s in SOURCES]
        subprocess.check_call(cmd)
        os.replace(tmp, LIB)
    return LIB


if __name__ == "__main__":
    print(build_library(force=True, verbose=True))
