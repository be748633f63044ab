"""Builds libcsr5.so (HIP, gfx950) in-tree with hipcc, no torch involved, and next to it _marshal.so, which takes torch's
tensors apart for the calls of a serving step."""
from __future__ import annotations

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


def build(verbose: bool = True, extra=()) -> str:
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
    build_marshal(verbose)
    return OUT


def build_marshal(verbose: bool = True) -> str:
    """_marshal.so, against this interpreter's and torch's headers."""
    import sysconfig

    import torch
    t = os.path.dirname(torch.__file__)
    tmp = MARSHAL + f".tmp{os.getpid()}"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", INC, "-I", os.path.join(t, "include"), "-I", os.path.join(t, "include", "torch", "csrc", "api", "include"),
           "-I", sysconfig.get_paths()["include"], MARSHAL_SRC, "-o", tmp, "-L", os.path.join(t, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10",
           "-L", PKG, "-l:libcsr5.so", "-Wl,-rpath,$ORIGIN"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.check_call(cmd, stdin=subprocess.DEVNULL)
    os.replace(tmp, MARSHAL)
    return MARSHAL


def is_stale() -> bool:
    if not os.path.exists(OUT) or not os.path.exists(MARSHAL):
        return True
    t = min(os.path.getmtime(OUT), os.path.getmtime(MARSHAL))
    deps = SRC + HEADERS + [MARSHAL_SRC] + [os.path.join(INC, "csr5.h")]
    return any(os.path.getmtime(d) > t for d in deps)


if __name__ == "__main__":
    build(extra=sys.argv[1:])
