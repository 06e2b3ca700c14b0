"""Compile the gfx950 HIP sources of this package into libvsa2.so, and the host
module _host.so that hands it torch tensors (both in-tree)."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIB = os.path.join(PKG, "libvsa2.so")
HOST = os.path.join(PKG, "_host.so")
OBJ = os.path.join(PKG, "_build")

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    # keep MFMA accumulators in VGPRs (fewer AGPR <-> VGPR copies in the attention loops)
    "-mllvm", "-amdgpu-mfma-vgpr-form",
    "-I", INCLUDE, "-I", CSRC,
]


def sources():
    return sorted(glob.glob(os.path.join(CSRC, "*.hip")))


def _host_flags():
    """g++ flags against this Python's torch (C++ headers and libraries)."""
    import torch
    root = os.path.dirname(torch.__file__)
    cxx = ["-O2", "-std=c++17", "-fPIC", "-Wall", "-D__HIP_PLATFORM_AMD__",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI), "-I", INCLUDE, "-I", "/opt/rocm/include",
           "-I", sysconfig.get_paths()["include"], "-isystem", os.path.join(root, "include")]
    # torch's own libraries are in the process before the module is loaded
    link = ["-L", os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10", "-L", PKG, "-lvsa2",
            "-Wl,-rpath,$ORIGIN"]
    return cxx, link


def build_host(stage: str) -> None:
    """Compile csrc/host.cpp ("compile") or link _host.so against libvsa2.so ("link")."""
    cxx, link = _host_flags()
    obj = os.path.join(OBJ, "host.cpp.o")
    tmp = HOST + ".tmp%d" % os.getpid()
    gxx = os.environ.get("CXX", "g++")
    cmd = [gxx, *cxx, "-c", os.path.join(CSRC, "host.cpp"), "-o", obj] if stage == "compile" else \
        [gxx, "-shared", "-o", tmp, obj, *link]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("%s of host.cpp failed:\n%s" % (stage, r.stderr))
    if stage == "link":
        os.replace(tmp, HOST)


def build(verbose: bool = False, jobs: int = 8) -> str:
    """Compile every csrc/*.hip for gfx950 and link libvsa2.so, then the host
    module.  Always recompiles (this is the build check); returns the library path."""
    os.makedirs(OBJ, exist_ok=True)
    srcs = sources()

    def compile_one(src):
        obj = os.path.join(OBJ, os.path.basename(src) + ".o")
        cmd = [HIPCC, *FLAGS, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError("hipcc failed for %s:\n%s" % (src, r.stderr))
        if verbose and r.stderr.strip():
            print(r.stderr)
        return obj

    with ThreadPoolExecutor(min(jobs, len(srcs) + 1)) as ex:
        host = ex.submit(build_host, "compile")
        objs = list(ex.map(compile_one, srcs))
        host.result()
    tmp = LIB + ".tmp%d" % os.getpid()
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs],
                       capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("link failed:\n" + r.stderr)
    os.replace(tmp, LIB)
    build_host("link")
    return LIB


if __name__ == "__main__":
    print(build(verbose=True))
