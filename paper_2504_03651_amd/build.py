"""Builds libecho.so in-tree with hipcc for gfx950, and the bindings' compiled part
_binding.so with g++ (no JIT, no cache).

``build_sanitized()`` builds a copy whose host code (the planner, the block
manager and the validation in the C ABI) carries AddressSanitizer and
UndefinedBehaviorSanitizer instrumentation, for running the host-only tests
under them on a CPU; the device code is built as usual."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
OUT = os.path.join(PKG, "libecho.so")
SOURCES = ["kernels.hip", "plan.cpp", "abi.cpp", "kvm.cpp", "layer.hip", "fp8.hip", "moe.hip",
           "int8.hip", "rope.hip", "norm.hip"]

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
FLAGS = ["--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall",
         # packed fp32 instructions stay off (see the design notes)
         "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", os.path.join(ROOT, "include"), "-I", CSRC]


BINDING = os.path.join(PKG, "_binding.so")


def _lacking() -> str | None:
    """What the compiled part of the bindings needs and is not here."""
    import shutil
    import sysconfig
    cxx = os.environ.get("CXX", "g++")
    if not shutil.which(cxx):
        return f"the host compiler {cxx}"
    if not os.path.exists(os.path.join(sysconfig.get_paths()["include"], "Python.h")):
        return "Python.h"
    try:
        import torch
    except ImportError:
        return "PyTorch"
    header = os.path.join(os.path.dirname(torch.__file__), "include", "torch", "csrc", "autograd", "python_variable.h")
    return None if os.path.exists(header) else "PyTorch's headers"


def build_binding(verbose: bool = False) -> str | None:
    """The compiled part of the Python bindings (host code only), against PyTorch's headers.
    The library itself needs neither those nor a host compiler: without them there is no
    such part, and the bindings that need it raise."""
    lacking = _lacking()
    if lacking:
        if os.path.exists(BINDING):
            os.remove(BINDING)
        sys.stderr.write(f"{os.path.basename(BINDING)} is not built, {lacking} is missing: "
                         "int8.py, rope.py and norm.py will raise\n")
        return None
    import sysconfig

    import torch
    root = os.path.dirname(torch.__file__)
    tmp = BINDING + ".tmp"
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}",
           "-I", os.path.join(ROOT, "include"), "-isystem", os.path.join(root, "include"),
           "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, "binding.cpp"), "-o", tmp,
           "-L" + os.path.join(root, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("g++ failed on binding.cpp")
    os.replace(tmp, BINDING)
    return BINDING


def build(verbose: bool = False) -> str:
    bdir = os.path.join(ROOT, "_build")
    os.makedirs(bdir, exist_ok=True)
    objs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src + ".o")
        cmd = [HIPCC, *FLAGS, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError(f"hipcc failed on {src}")
        objs.append(obj)
    tmp = OUT + ".tmp"
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", tmp, *objs,
           "-L/opt/rocm/lib", "-lhipblaslt", "-Wl,-rpath,/opt/rocm/lib"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link of libecho.so failed")
    os.replace(tmp, OUT)
    build_binding(verbose)
    return OUT


# host sources instrumented by build_sanitized(); the others keep device code
SANITIZED = ("plan.cpp", "abi.cpp", "kvm.cpp")
SAN_FLAGS = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g"]


def sanitizer_runtime() -> str:
    """The clang AddressSanitizer runtime that a sanitized build needs
    preloaded into an uninstrumented interpreter."""
    import glob
    hits = sorted(glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so"))
    if not hits:
        raise RuntimeError("clang AddressSanitizer runtime not found under /opt/rocm/llvm")
    return hits[-1]


def build_sanitized(out: str | None = None, verbose: bool = False) -> str:
    out = out or os.path.join(ROOT, "_build", "san", "libecho_san.so")
    bdir = os.path.dirname(out)
    os.makedirs(bdir, exist_ok=True)
    objs = []
    for src in SOURCES:
        obj = os.path.join(bdir, src + ".o")
        extra = SAN_FLAGS if src in SANITIZED else []
        cmd = [HIPCC, *FLAGS, *extra, "-c", os.path.join(CSRC, src), "-o", obj]
        if verbose:
            print(" ".join(cmd), flush=True)
        r = subprocess.run(cmd, capture_output=True, text=True)
        if r.returncode != 0:
            sys.stderr.write(r.stdout + r.stderr)
            raise RuntimeError(f"hipcc failed on {src} (sanitized build)")
        objs.append(obj)
    cmd = [HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Xarch_host", "-fsanitize=address",
           "-Xarch_host", "-fsanitize=undefined", "-shared-libsan", "-o", out, *objs,
           "-L/opt/rocm/lib", "-lhipblaslt", "-Wl,-rpath,/opt/rocm/lib"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        sys.stderr.write(r.stdout + r.stderr)
        raise RuntimeError("link of the sanitized libecho failed")
    return out


if __name__ == "__main__":
    print(build(verbose=True))
