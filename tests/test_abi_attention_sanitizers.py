"""The host code of the rotary, cache and attention calls under AddressSanitizer and UndefinedBehaviorSanitizer (CPU, no
GPU): tests/abi_attn_driver.cpp, built and run as the driver of the other calls is."""
import concurrent.futures as cf
import glob
import os
import subprocess

import pytest

from test_abi_sanitizers import CSRC, HIPCC, INCLUDE, ROOT, SAN, _run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_host_code_of_the_attention_calls(tmp_path):
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", *SAN,
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-fhip-fp32-correctly-rounded-divide-sqrt", "-I", INCLUDE, "-I", CSRC]
    srcs = sorted(glob.glob(os.path.join(CSRC, "*.hip")))
    objs = [str(tmp_path / (os.path.basename(s) + ".o")) for s in srcs]
    with cf.ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as ex:
        list(ex.map(_run, [[HIPCC, *flags, "-c", s, "-o", o] for s, o in zip(srcs, objs)]))
    drv = str(tmp_path / "driver.o")
    _run([HIPCC, "-x", "c++", "-O1", "-g", "-std=c++17", *SAN, "-I", INCLUDE, "-I", "/opt/rocm/include",
          "-D__HIP_PLATFORM_AMD__", "-c", os.path.join(ROOT, "tests", "abi_attn_driver.cpp"), "-o", drv])
    exe = str(tmp_path / "abi_attn_driver")
    _run([HIPCC, "--offload-arch=gfx950", *SAN, *objs, drv, "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    out = res.stdout + res.stderr
    assert res.returncode == 0, out[-4000:]
    assert "runtime error" not in out and "ERROR: AddressSanitizer" not in out and "LeakSanitizer" not in out
    assert " 0 failures" in out
