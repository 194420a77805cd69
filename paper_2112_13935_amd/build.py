"""Build the HIP libraries in-tree for gfx950: paper_2112_13935_amd/libaet_sgd.so (the rounds)
and libaet_ops.so (the operators)."""
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
INCLUDE = os.path.join(os.path.dirname(HERE), "include")

# packed-fp32 VALU forms are switched off for all device code of this library
HIPCC_FLAGS = ["-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-shared",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
               "-Wall", "-Wno-unused-function"]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def needs_build() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = sources() + glob.glob(os.path.join(CSRC, "*.h")) + [
        os.path.join(os.path.dirname(HERE), "include", "aet_sgd.h")]
    return any(os.path.getmtime(d) > t for d in deps)


def build(force: bool = True, verbose: bool = False) -> str:
    if not force and not needs_build():
        return LIB
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    cmd = [hipcc] + HIPCC_FLAGS + ["-o", LIB] + sources()
    if verbose:
        print(" ".join(cmd))
    subprocess.run(cmd, check=True)
    return LIB


def build_ops(verbose: bool = False) -> str:
    """The operators' library: a compilation per source, side by side, and a link."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [f for f in HIPCC_FLAGS if f != "-shared"] + ["-I", INCLUDE]
    objects = os.path.join(HERE, "_build")
    os.makedirs(objects, exist_ok=True)

    def one(src):
        obj = os.path.join(objects, os.path.basename(src)[:-len(".hip")] + ".o")
        cmd = [hipcc] + flags + ["-c", src, "-o", obj]
        if verbose:
            print(" ".join(cmd))
        subprocess.run(cmd, check=True)
        return obj

    with ThreadPoolExecutor(4) as pool:
        made = list(pool.map(one, sorted(glob.glob(os.path.join(OPS_CSRC, "*.hip")))))
    subprocess.run([hipcc, "--offload-arch=gfx950", "-fPIC", "-shared", "-o", OPS_LIB] + made, check=True)
    return OPS_LIB


if __name__ == "__main__":
    build(force=True, verbose=True)
    build_ops(verbose=True)
