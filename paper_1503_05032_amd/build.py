"""Builds libcsr5.so (HIP, gfx950) in-tree with hipcc, no torch involved, and next to it, where torch is installed,
_marshal.so, which takes torch's tensors apart for the calls of a serving step."""
from __future__ import annotations

import importlib.util
import os
import shutil
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
SRC = [os.path.join(PKG, "csrc", name) for name in ("csr5.hip", "experts.hip", "grouped.hip")]
HEADERS = [os.path.join(PKG, "csrc", name) for name in ("row_share.h", "far_lists.h", "numbers.h")]
INC = os.path.join(ROOT, "include")
OUT = os.path.join(PKG, "libcsr5.so")
MARSHAL_SRC = os.path.join(PKG, "csrc", "marshal.cpp")
MARSHAL = os.path.join(PKG, "_marshal.so")

FLAGS = [
    "-O3", "-std=c++17", "--offload-arch=gfx950", "-fPIC",
    "-munsafe-fp-atomics",            # hardware fp64 atomic add (memory is coarse-grained)
    # packed-fp32 instructions are switched off: some forms misbehave on this hardware
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-command-line-argument", "-Wno-unknown-attributes",
]


def hipcc() -> str:
    for c in (os.environ.get("HIPCC"), shutil.which("hipcc"), "/opt/rocm/bin/hipcc"):
        if c and os.path.exists(c):
            return c
    raise RuntimeError("hipcc not found")


def host_compiler() -> str:
    """A C++ compiler: the environment's, g++, or the one that hipcc itself uses."""
    near = os.path.join(os.path.dirname(os.path.realpath(hipcc())), "..", "lib", "llvm", "bin", "clang++")
    for c in (os.environ.get("CXX"), shutil.which("g++"), near):
        if c and shutil.which(c):
            return c
    raise RuntimeError("no C++ compiler found: set CXX")


def torch_there() -> bool:
    """Without torch nobody has tensors to take apart: the library alone is the build."""
    return importlib.util.find_spec("torch") is not None


def build(verbose: bool = True, extra=()) -> str:
    """The library, and _marshal.so where there is torch to build it with."""
    build_library(verbose, extra)
    if torch_there():
        build_marshal(verbose)
    return OUT


def build_library(verbose: bool = True, extra=()) -> str:
    """Compiles every source, side by side, and links them."""
    tmp = OUT + f".tmp{os.getpid()}"
    objects = [f"{tmp}.{os.path.basename(src)}.o" for src in SRC]

    def start(cmd):
        if verbose:
            print(" ".join(cmd), flush=True)
        return subprocess.Popen(cmd, stdin=subprocess.DEVNULL)

    try:
        running = [start([hipcc(), *FLAGS, *extra, "-I", INC, "-c", src, "-o", obj]) for src, obj in zip(SRC, objects)]
        codes = [p.wait() for p in running]
        if any(codes):
            raise subprocess.CalledProcessError(next(c for c in codes if c), running[0].args[0])
        if start([hipcc(), *FLAGS, *extra, "-shared", "-o", tmp, *objects]).wait():
            raise RuntimeError("linking libcsr5.so failed")
        os.replace(tmp, OUT)
    finally:
        for obj in objects:
            if os.path.exists(obj):
                os.remove(obj)
    return OUT


def build_marshal(verbose: bool = True) -> str:
    """_marshal.so, against this interpreter's and torch's headers."""
    import sysconfig

    import torch
    t = os.path.dirname(torch.__file__)
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = [host_compiler(), "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", INC, "-I", os.path.join(t, "include"), "-I", os.path.join(t, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], MARSHAL_SRC, "-o", tmp, "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-L", PKG, "-l:libcsr5.so", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd, stdin=subprocess.DEVNULL)
    os.replace(tmp, MARSHAL)
    return MARSHAL


def is_stale() -> bool:
    header = [os.path.join(INC, "csr5.h")]
    made = {OUT: SRC + HEADERS + header}
    if torch_there():
        made[MARSHAL] = [MARSHAL_SRC] + header
    return any(not os.path.exists(out) or any(os.path.getmtime(d) > os.path.getmtime(out) for d in deps) for out, deps in made.items())


if __name__ == "__main__":
    build(extra=sys.argv[1:])
