"""Build libmoe.so (the HIP kernels and the C ABI) in-tree for gfx950, and
_binding.so, the native Python binding of the attention calls, the norm and the
calls with 4-bit weights.

    python paper_2606_10493_amd/build.py

(run it by path: importing the package loads the library it builds).

Every .hip file under csrc/ is compiled with hipcc in parallel and linked
into paper_2606_10493_amd/libmoe.so.  It compiles on a machine without a
GPU (hipcc cross-compiles for gfx950).  csrc/binding.cpp is compiled with g++
against the Python and torch headers and linked with libmoe.so; where one of
these is missing the library is built all the same, and these calls
are left without their Python binding.
"""
from __future__ import annotations

import concurrent.futures as cf
import glob
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
LIB = os.path.join(PKG, "libmoe.so")
BINDING = os.path.join(PKG, "_binding.so")
ARCH = "gfx950"

HIPCC = os.environ.get("HIPCC", shutil.which("hipcc") or "/opt/rocm/bin/hipcc")
CXX = "g++"
PYTHON_INCLUDE = sysconfig.get_paths()["include"]

CFLAGS = [
    f"--offload-arch={ARCH}", "-O3", "-std=c++17", "-fPIC",
    "-fhip-fp32-correctly-rounded-divide-sqrt",
    # Packed fp32 VALU forms are kept out of the generated code.
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-Wall", "-Wno-unused-function",
    # A loop transformation that was asked for and not done is an error.
    "-Werror=pass-failed",
    "-I", INCLUDE, "-I", CSRC,
]


def _compile(src: str) -> str:
    obj = os.path.join(BUILD_DIR, os.path.basename(src) + ".o")
    cmd = [HIPCC, *CFLAGS, "-c", src, "-o", obj]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"hipcc failed on {src}:\n{res.stdout}\n{res.stderr}")
    return obj


def build_binding() -> bool:
    """_binding.so, if there is what it needs; otherwise none, since an earlier one might not fit the library."""
    if os.path.exists(BINDING):
        os.remove(BINDING)
    missing = None
    if not (CXX and shutil.which(CXX)):
        missing = f"C++ compiler {CXX}"
    elif not os.path.exists(os.path.join(PYTHON_INCLUDE, "Python.h")):
        missing = f"{PYTHON_INCLUDE}/Python.h"
    try:
        import torch  # its headers and its ABI flag
    except ImportError:
        missing = "torch"
    if missing:
        print("_binding.so is not built, the attention calls, the norm and the calls with 4-bit weights have no Python "
              f"binding: {missing} is missing", file=sys.stderr)
        return False
    lib_dir = os.path.join(os.path.dirname(torch.__file__), "lib")
    include = os.path.join(os.path.dirname(torch.__file__), "include")
    tmp = BINDING + ".tmp"
    cmd = [CXX, "-O2", "-std=c++17", "-fPIC", "-shared", "-Wall", "-D__HIP_PLATFORM_AMD__", "-DUSE_ROCM",
           f"-D_GLIBCXX_USE_CXX11_ABI={int(torch._C._GLIBCXX_USE_CXX11_ABI)}", "-I", INCLUDE, "-isystem", include,
           "-isystem", os.path.join(include, "torch", "csrc", "api", "include"),
           "-isystem", PYTHON_INCLUDE, "-isystem", "/opt/rocm/include",
           os.path.join(CSRC, "binding.cpp"), "-o", tmp,
           "-L", PKG, "-lmoe", "-L", lib_dir, "-ltorch_python", "-ltorch_cpu", "-lc10", "-lc10_hip", "-Wl,-rpath,$ORIGIN"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"building binding.cpp failed:\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, BINDING)
    return True


def build(verbose: bool = False) -> str:
    os.makedirs(BUILD_DIR, exist_ok=True)
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    with cf.ThreadPoolExecutor(max_workers=min(8, len(srcs))) as ex:
        objs = list(ex.map(_compile, srcs))
    tmp = LIB + ".tmp"
    cmd = [HIPCC, f"--offload-arch={ARCH}", "-shared", "-fPIC", *objs, "-o", tmp]
    res = subprocess.run(cmd, capture_output=True, text=True)
    if res.returncode != 0:
        raise RuntimeError(f"link failed:\n{res.stdout}\n{res.stderr}")
    os.replace(tmp, LIB)
    bound = build_binding()
    if verbose:
        print(f"built {LIB} from {len(srcs)} sources" + (f", and {BINDING}" if bound else ""))
    return LIB


if __name__ == "__main__":
    build(verbose=True)
    sys.exit(0)
