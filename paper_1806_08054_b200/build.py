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


def marshal_path() -> str:
    """The binding's compiled marshalling: it has torch's and Python's memory layouts in it, so its name says
    which ones, and a file that was built for others is not looked at."""
    import sysconfig
    import torch
    return os.path.join(_HERE, "_marshal-torch%s-%s%s" % (torch.__version__, (torch.version.git_version or "")[:8],
                                                          sysconfig.get_config_var("EXT_SUFFIX") or ".so"))


def load_marshal():
    """The module from that file; ImportError where there is none."""
    import importlib.util
    import sys
    name = os.path.basename(_HERE) + "._marshal"
    if name not in sys.modules:
        path = marshal_path()
        if not os.path.exists(path):
            raise ImportError("not built: " + path)
        spec = importlib.util.spec_from_file_location(name, path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        sys.modules[name] = module
    return sys.modules[name]


def build_marshal(force: bool = False) -> bool:
    """Compile the binding's argument marshalling (``csrc/ecq_marshal.cpp``) next to this file.  Where that cannot
    be done (no headers of Python or torch) the binding does the same in Python, a few microseconds a call slower."""
    source, target = os.path.join(CSRC, "ecq_marshal.cpp"), marshal_path()
    if force or not os.path.exists(target) or os.path.getmtime(target) < os.path.getmtime(source):
        import sysconfig
        import torch
        libs = os.path.join(os.path.dirname(torch.__file__), "lib")  # loaded by torch before this is
        base = os.path.join(os.path.dirname(torch.__file__), "include")
        tmp = target + ".tmp.%d" % os.getpid()
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
        os.replace(tmp, target)
    try:
        load_marshal()
    except ImportError as e:
        print("ecq_marshal.cpp is built and not loaded: %s" % e)
        return False
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
