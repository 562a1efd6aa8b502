"""Build the HIP library ``libtre.so`` for gfx950 with hipcc, and the binding's
``_tensors.so`` (in-tree)."""
from __future__ import annotations

import concurrent.futures as cf
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OBJ = os.path.join(HERE, "_build")
LIB = os.path.join(HERE, "libtre.so")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
ARCH = "gfx950"
FLAGS = [
    "-O3", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}",
    # keep the compiler from forming packed fp32 instructions
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-Wall", "-Wno-unused-function",
    # the LDS copies' assembly sets m0 and says so; clang warns at every use
    # that the clobber list names a reserved register
    "-Wno-inline-asm",
]


def sources():
    return sorted(os.path.join(CSRC, f) for f in os.listdir(CSRC) if f.endswith((".hip", ".cpp")))


def _compile(src: str) -> str:
    obj = os.path.join(OBJ, os.path.basename(src) + ".o")
    cmd = [HIPCC, *FLAGS, "-c", src, "-o", obj]
    if src.endswith(".hip"):
        cmd[1:1] = ["-x", "hip"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stderr}")
    return obj


TENSORS = os.path.join(HERE, "_tensors.so")


def build_tensors() -> str:
    """Build ``_tensors.so``, the binding's reader of lists of torch tensors: host
    code against torch's headers, the only part that knows them."""
    import sysconfig

    import torch
    from torch.utils import cpp_extension

    dirs = [*cpp_extension.include_paths(), sysconfig.get_paths()["include"]]
    libs = cpp_extension.library_paths()
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-w", *(f"-I{d}" for d in dirs),
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", os.path.join(HERE, "pysrc", "tensors.cpp"),
           "-o", TENSORS + ".tmp", *(f"-L{d}" for d in libs), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    try:
        r = subprocess.run(cmd, capture_output=True, text=True)
    except OSError as e:
        raise RuntimeError(f"{os.path.basename(TENSORS)}: no C++ compiler: {e}") from None
    if r.returncode != 0:
        raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stderr}")
    os.replace(TENSORS + ".tmp", TENSORS)
    return TENSORS


def build(verbose: bool = False, binding: bool = True) -> str:
    """Build ``libtre.so``, for which hipcc is enough, and ``_tensors.so``, for
    which torch, Python's headers and a C++ compiler are needed: the library is
    linked also where that fails, and without torch only a note is left."""
    os.makedirs(OBJ, exist_ok=True)
    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        reader = ex.submit(build_tensors) if binding else None
        objs = list(ex.map(_compile, sources()))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-o", tmp, *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stderr}")
    os.replace(tmp, LIB)
    if verbose:
        print(f"built {LIB}")
    try:
        if reader:
            reader.result()
    except ImportError as e:
        print(f"{os.path.basename(TENSORS)}, the Python binding's reader of tensors, is not built: {e}", file=sys.stderr)
    return LIB


SAN_LIB = os.path.join(HERE, "libtre_host_san.so")
SAN_OBJ = os.path.join(HERE, "_build_san")
# AddressSanitizer + UBSan on the host code only (-Xarch_host keeps them off
# the gfx950 device pass, which is built as usual), linked against the
# compiler's shared sanitizer runtime
SAN_FLAGS = [
    "-O1", "-g", "-std=c++17", "-fPIC", f"--offload-arch={ARCH}", "-fno-omit-frame-pointer",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
    "-Xarch_host", "-shared-libsan", "-I", os.path.join(ROOT, "include"),
]


def build_host_sanitized(verbose: bool = False) -> str:
    """Build ``libtre_host_san.so``: the library with its host code (plan
    parsing, classification, workspace layout, argument checks, launch
    set-up) under AddressSanitizer and UBSan, for the CPU tests
    (``tests/sanitize.sh``); never loaded unless TRE_HOST_SANITIZED=1."""
    os.makedirs(SAN_OBJ, exist_ok=True)

    def one(src):
        obj = os.path.join(SAN_OBJ, os.path.basename(src) + ".o")
        cmd = [HIPCC, "-x", "hip", *SAN_FLAGS, "-c", src, "-o", obj]
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            raise RuntimeError(f"compile failed: {' '.join(cmd)}\n{r.stderr}")
        return obj

    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        objs = list(ex.map(one, sources()))
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", "-Xarch_host", "-fsanitize=address,undefined",
           "-Xarch_host", "-shared-libsan", "-o", SAN_LIB + ".tmp", *objs]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"link failed: {' '.join(cmd)}\n{r.stderr}")
    os.replace(SAN_LIB + ".tmp", SAN_LIB)
    if verbose:
        print(f"built {SAN_LIB}")
    return SAN_LIB


if __name__ == "__main__":
    if "--host-sanitized" in sys.argv:
        build_host_sanitized(verbose=True)
    else:
        build(verbose=True, binding="--library" not in sys.argv)
    sys.exit(0)
