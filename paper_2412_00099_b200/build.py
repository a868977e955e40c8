"""Builds libmcce.so (CUDA, sm_100a only) and _marshal.so next to this file:  python -m paper_2412_00099_b200.build

libmcce.so needs nvcc alone.  _marshal.so, the torch side of the operators' binding, needs g++ and the headers of torch, Python
and CUDA as well; where it cannot be built the library is built all the same and only those operators are missing from
the binding, which says so when they are called."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys
import sysconfig
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libmcce.so")
MARSHAL = os.path.join(HERE, "_marshal.so")
SOURCES = ["api.cu", "route.cu", "route_thread.cu", "route_static.cu", "route_gemm.cu", "route_gemm_res.cu", "route_fused.cu", "belady.cu", "group.cu", "ffn_simt.cu", "ffn_tc.cu", "norm.cu", "rows.cu", "gen.cu"]
NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-Xcompiler", "-fPIC,-Wall", "-I", INCLUDE, "-I", CSRC]


def _newest(paths):
    return max(os.path.getmtime(p) for p in paths)


def build(force: bool = False, verbose: bool = False) -> str:
    srcs = [os.path.join(CSRC, s) for s in SOURCES]
    deps = srcs + [os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".cuh", ".h"))] + [
        os.path.join(INCLUDE, "mcce.h")]
    if force or not os.path.exists(LIB) or os.path.getmtime(LIB) < _newest(deps):
        _build_library(srcs, verbose)
    try:
        marshal = build_marshal(force)
        if verbose:
            sys.stderr.write("%s\n" % marshal)
    except (RuntimeError, OSError, ImportError) as e:
        sys.stderr.write("_marshal.so was not built (the binding's operators around the experts will be missing): %s\n" % e)
    return LIB


def _build_library(srcs, verbose):
    os.makedirs(OBJ, exist_ok=True)
    nvcc = os.environ.get("NVCC", "nvcc")

    def compile_one(src):
        obj = os.path.join(OBJ, os.path.basename(src) + ".o")
        cmd = [nvcc, *NVCC_FLAGS, "-c", src, "-o", obj] + (["-Xptxas", "-v"] if verbose else [])
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("nvcc failed for %s:\n%s" % (src, r.stderr))
        if verbose:
            sys.stderr.write(r.stderr)
        return obj

    with ThreadPoolExecutor(len(srcs)) as ex:
        objs = list(ex.map(compile_one, srcs))
    subprocess.check_call([nvcc, "-shared", "-o", LIB, *objs, "-gencode", "arch=compute_100a,code=sm_100a"])


def marshal_target() -> str:
    """What _marshal.so has to be built for: it uses the C++ interface of torch and the C interface of Python."""
    import torch
    return "torch %s, %s" % (torch.__version__, sysconfig.get_config_var("SOABI"))


def _cuda_home() -> str:
    nvcc = shutil.which(os.environ.get("NVCC", "nvcc"))
    homes = [os.path.dirname(os.path.dirname(os.path.realpath(nvcc)))] if nvcc else []
    homes += [h for h in (os.environ.get("CUDA_HOME"), "/usr/local/cuda") if h]
    for h in homes:
        if os.path.exists(os.path.join(h, "include", "cuda_runtime_api.h")):
            return h
    raise RuntimeError("no CUDA headers: neither nvcc on the path nor CUDA_HOME leads to them")


def build_marshal(force: bool = False) -> str:
    """Builds _marshal.so, the torch side of the operators' binding (host code: g++ against torch's own headers).  It is out of date
    when its sources are newer or when it was built for another torch or Python."""
    src, header = os.path.join(CSRC, "marshal.cpp"), os.path.join(INCLUDE, "mcce.h")
    target, stamp = marshal_target(), os.path.join(OBJ, "marshal.txt")
    if not force and os.path.exists(MARSHAL) and os.path.exists(stamp) and os.path.getmtime(MARSHAL) >= _newest([src, header]):
        with open(stamp) as f:
            if f.read() == target:
                return MARSHAL
    import torch
    home, cuda = os.path.dirname(torch.__file__), _cuda_home()
    includes = [INCLUDE, os.path.join(home, "include"), os.path.join(home, "include", "torch", "csrc", "api", "include"),
                sysconfig.get_paths()["include"], os.path.join(cuda, "include")]
    cmd = ["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
           "-DMCCE_BUILT_FOR=\"%s\"" % target,
           *[x for i in includes for x in ("-isystem" if i != INCLUDE else "-I", i)], src, "-o", MARSHAL + ".new",
           "-L" + os.path.join(home, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10_cuda", "-lc10"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("g++ failed for marshal.cpp:\n%s" % r.stderr)
    os.makedirs(OBJ, exist_ok=True)
    os.replace(MARSHAL + ".new", MARSHAL)
    with open(stamp, "w") as f:
        f.write(target)
    return MARSHAL


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    build_marshal()
