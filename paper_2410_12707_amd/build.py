"""Builds libadatopk.so (HIP kernels + C ABI) for gfx950 with hipcc, in-tree, and next to it
libadatopk_measure.so: the same sources compiled with ADATOPK_MEASURE_BUILD, which adds the
benchmark-only hooks of include/adatopk_measure.h (per-kernel dispatch timing, plain streaming
kernels).  The product library carries none of them.  _marshal is the Python extension that reads
the arguments and makes the calls (marshal.cpp, host code only); the package works without it."""
from __future__ import annotations

import glob
import os
import subprocess
import sysconfig
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
LIB = os.path.join(HERE, "libadatopk.so")
MEASURE_LIB = os.path.join(HERE, "libadatopk_measure.so")
# (the suffix names the Python it is built for: another one does not load it)
MARSHAL_LIB = os.path.join(HERE, "_marshal" + (sysconfig.get_config_var("EXT_SUFFIX") or ".so"))
MARSHAL_SOURCE = os.path.join(CSRC, "marshal.cpp")
HEADER = os.path.join(ROOT, "include", "adatopk.h")
SOURCES = [os.path.join(CSRC, name) for name in ("adatopk.hip", "act8.hip", "layernorm.hip", "rmsnorm.hip", "weight_grad.hip", "fp8.hip", "fp8_product.hip", "muon.hip",
                                             "adatopk_host.cpp")]
INTERNAL_HEADERS = [os.path.join(CSRC, name) for name in ("wire_layout.h", "act8_layout.h", "fp8_layout.h", "stage_ops.h", "norm.h", "fp8_form.h", "row_tiles.h")]

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Wall", "-Wextra",
    # packed-fp32 instruction forms are kept out of the generated code on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-I", os.path.join(ROOT, "include"), "-I", CSRC,
]


def build_library(verbose: bool = False, out: str = LIB, defines=()) -> str:
    """Compiles the library to `out`, its sources side by side; `defines` are extra -D macros (launch-shape overrides)."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    with tempfile.TemporaryDirectory() as scratch:
        objects = [os.path.join(scratch, os.path.basename(source) + ".o") for source in SOURCES]
        commands = [[hipcc] + HIPCC_FLAGS + ["-D" + d for d in defines] + ["-c", "-o", o, source] for o, source in zip(objects, SOURCES)]
        link = [hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", out] + objects
        if verbose:
            print("\n".join(" ".join(cmd) for cmd in commands + [link]), flush=True)
        running = [subprocess.Popen(cmd) for cmd in commands]
        failed = [cmd for cmd, code in [(p.args, p.wait()) for p in running] if code != 0]
        if failed:
            raise subprocess.CalledProcessError(1, failed[0])
        subprocess.run(link, check=True)
    return out


def build_measure_library(verbose: bool = False) -> str:
    return build_library(verbose, MEASURE_LIB, ("ADATOPK_MEASURE_BUILD",))


def build_marshal(verbose: bool = False) -> str:
    """The Python extension that reads the arguments and makes the calls (host code only)."""
    import torch

    base = os.path.dirname(torch.__file__)
    cmd = [os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-fvisibility=hidden",
           "-D_GLIBCXX_USE_CXX11_ABI=%d" % int(torch._C._GLIBCXX_USE_CXX11_ABI),
           "-isystem", os.path.join(base, "include"), "-isystem", os.path.join(base, "include", "torch", "csrc", "api", "include"),
           "-isystem", sysconfig.get_paths()["include"], "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Wall", "-Wextra", "-o", MARSHAL_LIB, MARSHAL_SOURCE,
           "-L" + os.path.join(base, "lib"), "-ltorch_python", "-ltorch_cpu", "-lc10"]
    if verbose:
        print(" ".join(cmd), flush=True)
    subprocess.run(cmd, check=True)
    return MARSHAL_LIB


def library_is_stale() -> bool:
    if not os.path.exists(LIB):
        return True
    t = os.path.getmtime(LIB)
    deps = SOURCES + [HEADER, os.path.join(ROOT, "include", "adatopk_measure.h")] + INTERNAL_HEADERS
    return any(os.path.getmtime(d) > t for d in deps)


def marshal_is_stale() -> bool:
    if not os.path.exists(MARSHAL_LIB):
        return True
    t = os.path.getmtime(MARSHAL_LIB)
    # it calls the library's functions by address, as the header declares them, and sizes buffers by the headers beside its source
    beside = glob.glob(os.path.join(os.path.dirname(MARSHAL_SOURCE), "*.h"))
    return any(os.path.getmtime(d) > t for d in [MARSHAL_SOURCE, HEADER] + beside)


if __name__ == "__main__":
    print(build_library(verbose=True))
    print(build_measure_library(verbose=True))
    print(build_marshal(verbose=True))
