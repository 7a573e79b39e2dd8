"""Build libsoftsync_ps.so (the C-ABI library with its sm_100a kernels) in-tree with nvcc, and the _marshal extension (argument checks and
output tensors of learn.py over torch's C++ tensors) with the host compiler."""
from __future__ import annotations

import hashlib
import os
import shutil
import subprocess
import sysconfig
import warnings

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsoftsync_ps.so")
SOURCES = ["softsync_ps.cu", "tensor_list.cu", "token_loss.cu"]
HEADERS = [os.path.join(CSRC, h) for h in ("update_kernels.cuh", "tensor_kernels.cuh", "token_kernels.cuh", "packed.cuh", "host_util.h")] + \
          [os.path.join(os.path.dirname(HERE), "include", h) for h in ("softsync_ps.h", "softsync_learn.h")]

NVCC_FLAGS = ["-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
              "-shared", "-Xcompiler", "-fPIC", "-cudart", "static", "--threads", "0"]


def nvcc() -> str:
    exe = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(exe):
        raise RuntimeError("nvcc not found: the library cannot be built")
    return exe


STAMP = LIB + ".hash"            # digest of the sources and flags the library was built from


def source_digest() -> str:
    h = hashlib.sha256(" ".join(NVCC_FLAGS).encode())
    for path in [os.path.join(CSRC, s) for s in SOURCES] + HEADERS:
        with open(path, "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def is_stale() -> bool:
    """True unless the library exists and was built from exactly the present sources (file times are not
    trusted: a copied tree does not keep them)."""
    return _stale(LIB, STAMP, source_digest)


def _stale(target: str, stamp: str, digest) -> bool:
    if not os.path.exists(target) or not os.path.exists(stamp):
        return True
    with open(stamp) as f:
        return f.read().strip() != digest()


# ---- the _marshal extension ----------------------------------------------------
MARSHAL = os.path.join(HERE, "_marshal.so")
MARSHAL_STAMP = MARSHAL + ".hash"
MARSHAL_SOURCES = [os.path.join(CSRC, "marshal.cpp")] + [os.path.join(os.path.dirname(HERE), "include", h) for h in ("softsync_ps.h", "softsync_learn.h")]
MARSHAL_FLAGS = ["-O2", "-std=c++17", "-shared", "-fPIC", "-fvisibility=hidden"]


def marshal_digest() -> str:
    import torch
    h = hashlib.sha256(" ".join(MARSHAL_FLAGS + [torch.__version__, sysconfig.get_python_version()]).encode())
    for path in MARSHAL_SOURCES:
        with open(path, "rb") as f:
            h.update(f.read())
    return h.hexdigest()


def build_marshal(force: bool = False) -> str:
    if not force and not _stale(MARSHAL, MARSHAL_STAMP, marshal_digest):
        return MARSHAL
    import torch
    root = os.path.dirname(torch.__file__)
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(nvcc())))
    include = [sysconfig.get_paths()["include"], os.path.join(root, "include"), os.path.join(root, "include", "torch", "csrc", "api", "include"),
               os.path.join(cuda, "include")]
    libs = os.path.join(root, "lib")
    cmd = [shutil.which("g++") or "g++"] + MARSHAL_FLAGS + ["-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI)]
    cmd += ["-isystem" + i for i in include] + ["-o", MARSHAL, MARSHAL_SOURCES[0], "-L" + libs, "-Wl,-rpath," + libs,
                                                "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_cuda"]
    for old in (MARSHAL_STAMP, MARSHAL):         # an extension of other sources must not be loaded if this fails
        if os.path.exists(old):
            os.remove(old)
    subprocess.run(cmd, check=True)
    with open(MARSHAL_STAMP, "w") as f:
        f.write(marshal_digest() + "\n")
    return MARSHAL


def build_library(force: bool = False, verbose: bool = False) -> str:
    if not force and not is_stale():
        return LIB
    cmd = [nvcc()] + NVCC_FLAGS + (["-Xptxas", "-v"] if verbose else []) + \
          ["-o", LIB] + [os.path.join(CSRC, s) for s in SOURCES]
    if os.path.exists(STAMP):
        os.remove(STAMP)
    subprocess.run(cmd, check=True)
    with open(STAMP, "w") as f:
        f.write(source_digest() + "\n")
    return LIB


def build(force: bool = False, verbose: bool = False) -> str:
    """Builds the library, then the extension; raises if either fails."""
    lib = build_library(force, verbose)
    build_marshal(force)
    return lib


def ensure_built() -> str:
    """Build the library and the extension if they are missing or were built from other sources.  A failed rebuild of the library raises: a
    library that does not match the header and the binding must not be loaded.  One of the extension warns: the server needs
    nothing of it, and what does raises when it is used."""
    lib = build_library()
    try:
        build_marshal()
    except (OSError, RuntimeError, subprocess.CalledProcessError) as e:
        warnings.warn("the _marshal extension could not be built (%s): the operators of learn.py are not available" % e)
    return lib


if __name__ == "__main__":
    import sys
    print(build(force=True, verbose="-v" in sys.argv))
