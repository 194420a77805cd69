"""Build in-tree for gfx950: paper_2112_13935_amd/libaet_sgd.so (the rounds), libaet_ops.so (the
operators) and _ops_torch.so (their binding to tensors)."""
from __future__ import annotations

import glob
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libaet_sgd.so")
OPS_CSRC = os.path.join(CSRC, "ops")
OPS_LIB = os.path.join(HERE, "libaet_ops.so")
OPS_TORCH = os.path.join(HERE, "_ops_torch.so")
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

# packed-fp32 VALU forms are switched off for all device code of this library
HIPCC_FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wall", "-Wno-unused-function"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _older(libs, deps) -> bool:
    if not all(os.path.exists(lib) for lib in libs):
        return True
    t = min(os.path.getmtime(lib) for lib in libs)
    return any(os.path.getmtime(d) > t for d in deps)


def needs_build() -> bool:
    return _older([LIB], sources() + glob.glob(os.path.join(CSRC, "*.h")) + [os.path.join(INCLUDE, "aet_sgd.h")])


def needs_build_ops() -> bool:
    """Whether the operators' library or its binding is missing or older than what it is made from."""
    return _older([OPS_LIB, OPS_TORCH], [f for d in (CSRC, OPS_CSRC, INCLUDE) for f in glob.glob(os.path.join(d, "*.h"))]
                  + glob.glob(os.path.join(OPS_CSRC, "*.hip")) + glob.glob(os.path.join(OPS_CSRC, "*.cpp")))


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc] + HIPCC_FLAGS + ["-o", LIB] + sources()
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    return LIB


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)


def build_ops(verbose: bool = False) -> str:
    """The operators' library (a compilation per source, side by side, and a link), and its binding."""
    from torch.utils import cpp_extension
    import sysconfig
    import torch
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f != "-shared"] + ["-I", INCLUDE]
    objects = os.path.join(HERE, "_build")
    os.makedirs(objects, exist_ok=True)
    torch_obj = os.path.join(objects, "ops_torch.o")
    headers = [h for d in cpp_extension.include_paths() + [sysconfig.get_paths()["include"]] for h in ("-isystem", d)]
    jobs = {os.path.join(objects, os.path.basename(src)[:-len(".hip")] + ".o"): [hipcc] + flags + ["-c", src]
            for src in sorted(glob.glob(os.path.join(OPS_CSRC, "*.hip")))}
    made = list(jobs)
    jobs[torch_obj] = ["g++", "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall",
                       f"-D_GLIBCXX_USE_CXX11_ABI={int(torch.compiled_with_cxx11_abi())}",
                       "-DTORCH_EXTENSION_NAME=_ops_torch", "-I", INCLUDE, *headers, "-c",
                       os.path.join(OPS_CSRC, "ops_torch.cpp")]
    with ThreadPoolExecutor(4) as pool:
        list(pool.map(lambda obj: _run(jobs[obj] + ["-o", obj], verbose), jobs))
    _run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-Wl,-soname,libaet_ops.so", "-o", OPS_LIB] + made, verbose)
    libs = [a for d in cpp_extension.library_paths() for a in ("-L" + d,)]
    _run(["g++", "-shared", "-o", OPS_TORCH, torch_obj, OPS_LIB, *libs, "-lc10", "-ltorch", "-ltorch_cpu", "-ltorch_python",
          "-Wl,-rpath,$ORIGIN"], verbose)
    return OPS_LIB


if __name__ == "__main__":
    build(force=True, verbose=True)
    build_ops(verbose=True)
