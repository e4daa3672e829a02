"""Build the HIP libraries (gfx950) and the binding's native parts in-tree: paper_2602_15318_amd/libsparrow.so,
libsparrow_paged.so, libsparrow_serve.so, _native.so, _native_paged.so, _native_serve.so."""
from __future__ import annotations

import concurrent.futures
import glob
import importlib.util
import os
import subprocess
import sys
import sysconfig

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libsparrow.so")
PAGED = os.path.join(HERE, "libsparrow_paged.so")
SERVE = os.path.join(HERE, "libsparrow_serve.so")
NATIVE = os.path.join(HERE, "_native.so")
NATIVE_PAGED = os.path.join(HERE, "_native_paged.so")
NATIVE_SERVE = os.path.join(HERE, "_native_serve.so")

# The preload count puts the leading scalar arguments of a kernel into scalar registers at launch: a
# wavefront's first load waits for no load of arguments (0.3 to 0.4 us on kernels of 6 to 13 us).
HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function", "-Wno-inline-asm",
]


def _run(cmd, verbose: bool) -> None:
    if verbose:
        print(" ".join(cmd), flush=True)
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    out = "\n".join(l for l in res.stdout.splitlines()
                    if "packed-fp32-ops" not in l)   # the host pass does not know the feature
    if res.returncode != 0:
        raise RuntimeError(f"{cmd[0]} failed:\n" + out)
    if verbose and out.strip():
        print(out)


def build(verbose: bool = False, extra=()) -> str:
    """Compile every csrc/*.hip into one shared library, csrc/paged/*.hip and csrc/serve/*.hip into others, and the binding's
    native part of each.  Always recompiles."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def hip(lib, *under):
        srcs = sorted(glob.glob(os.path.join(CSRC, *under, "*.hip")))
        _run([hipcc, *HIPCC_FLAGS, *extra, "-o", lib, *srcs], verbose)

    def native(lib, *source):
        torch = os.path.dirname(importlib.util.find_spec("torch").origin)
        _run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall",
              "-isystem", os.path.join(torch, "include"), "-isystem", os.path.join(torch, "include", "torch", "csrc", "api", "include"),
              "-isystem", sysconfig.get_paths()["include"], os.path.join(CSRC, *source), "-o", lib,
              "-L" + os.path.join(torch, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"], verbose)

    with concurrent.futures.ThreadPoolExecutor(6) as pool:     # side by side: each is one compiler, file after file
        for done in [pool.submit(hip, LIB), pool.submit(hip, PAGED, "paged"), pool.submit(hip, SERVE, "serve"), pool.submit(native, NATIVE, "binding.cpp"),
                     pool.submit(native, NATIVE_PAGED, "paged", "binding_paged.cpp"), pool.submit(native, NATIVE_SERVE, "serve", "binding_serve.cpp")]:
            done.result()
    return LIB


if __name__ == "__main__":
    print(build(verbose=True, extra=sys.argv[1:]))
