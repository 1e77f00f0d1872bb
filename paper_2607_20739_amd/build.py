"""Build libpgc.so (the C-ABI library of include/pgc.h and pgc_ops.h) for gfx950 with hipcc, and the
Python module that calls its operators on torch's tensors with g++.

Usage: python -m paper_2607_20739_amd.build   (or build() from Python)

Every HIP and C++ source under csrc/ is compiled with
  --offload-arch=gfx950 -O3 -std=c++17 -fPIC
  -Xclang -target-feature -Xclang -packed-fp32-ops
(the last pair keeps the compiler from emitting packed fp32 VALU instructions;
the host pass reports the feature as unknown, which is harmless and not shown;
other warnings go to stderr) and linked
into paper_2607_20739_amd/libpgc.so next to this file, linked against ROCm's
roctx library for the per-step profiler ranges.  binding/pgc_ops_torch.cpp becomes
paper_2607_20739_amd/_ops_torch.so, linked against that library and the installed torch; where
there is none, the library is built alone.
"""

import concurrent.futures
import importlib.util
import os
import shutil
import subprocess
import sys
import sysconfig

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
BUILD_DIR = os.path.join(ROOT, "_build")
LIB = os.path.join(PKG, "libpgc.so")
BINDING = os.path.join(PKG, "binding", "pgc_ops_torch.cpp")
BINDING_LIB = os.path.join(PKG, "_ops_torch.so")
SOURCES = sorted(f for f in os.listdir(CSRC) if f.endswith((".cpp", ".hip")))
ARCH = "gfx950"
ROCM_LIB = "/opt/rocm/lib"   # librocprofiler-sdk-roctx (per-step profiler ranges)


def hipcc():
    path = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(path):
        raise RuntimeError("hipcc not found: the HIP library cannot be built")
    return path


def common_flags():
    return ["--offload-arch=" + ARCH, "-O3", "-std=c++17", "-fPIC", "-Wall",
            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
            "-I", INCLUDE, "-I", CSRC]


def warnings(stderr):
    """The compiler's warnings but for the host pass's about the feature it does not know."""
    return [line for line in stderr.splitlines() if "warning" in line and "packed-fp32-ops" not in line
            and not line.endswith("generated when compiling for host.")
            and not line.endswith("generated when compiling for %s." % ARCH)]


def binding_flags():
    import torch
    include = os.path.join(os.path.dirname(torch.__file__), "include")
    return ["-O2", "-std=c++17", "-fPIC", "-Wall", "-D_GLIBCXX_USE_CXX11_ABI=%d" % torch._C._GLIBCXX_USE_CXX11_ABI,
            "-isystem", include, "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
            "-isystem", sysconfig.get_paths()["include"], "-I", INCLUDE]


def _run(what, cmd):
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError("%s failed:\n%s\n%s" % (what, " ".join(cmd), res.stderr))
    for line in warnings(res.stderr):
        print(line, file=sys.stderr)


def _compile(src):
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = ["g++"] + binding_flags() if src == BINDING else [hipcc()] + common_flags()
    _run("compiling " + src, cmd + ["-c", os.path.join(CSRC, src), "-o", obj])
    return obj


def _link(what, lib, cmd):
    tmp = lib + ".tmp"
    _run("linking " + what, cmd + ["-shared", "-fPIC", "-o", tmp])
    os.replace(tmp, lib)


def _link_library(objs):
    _link("libpgc.so", LIB, [hipcc(), "--offload-arch=" + ARCH] + objs +
          ["-L" + ROCM_LIB, "-Wl,-rpath," + ROCM_LIB, "-lrocprofiler-sdk-roctx"])


def _link_binding(obj):
    import torch
    torch_lib = os.path.join(os.path.dirname(torch.__file__), "lib")
    _link("_ops_torch.so", BINDING_LIB, ["g++", obj, "-L" + PKG, "-lpgc", "-Wl,-rpath,$ORIGIN", "-L" + torch_lib,
                                         "-lc10", "-ltorch_cpu", "-ltorch_hip", "-ltorch_python"])


def build(verbose=False):
    """Compile and link libpgc.so, then the torch binding; returns libpgc.so's path.

    The library needs no torch: it is there also where the binding cannot be built, which raises.  Without
    torch there is nothing to bind, and the binding is left out.
    """
    os.makedirs(BUILD_DIR, exist_ok=True)
    bind = importlib.util.find_spec("torch") is not None
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES) + 1) as pool:
        binding = pool.submit(_compile, BINDING) if bind else None
        _link_library(list(pool.map(_compile, SOURCES)))
        if verbose:
            print("built", LIB)
        if bind:
            _link_binding(binding.result())
    if verbose:
        print("built " + BINDING_LIB if bind else "no torch: %s is left out" % BINDING_LIB)
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
