"""The paged cache's host code under AddressSanitizer and UBSan, on the CPU, as test_abi_sanitized.py does it for
the eviction: both sanitizers on the host side only, driven by tests/cache_abi_sanitize_driver.cpp.  Skipped where a
GPU is visible: the driver's fake device pointers are for a runtime that has no device."""
import concurrent.futures as cf
import os

import pytest
import torch

import test_abi_sanitized as base

SOURCES = base.SOURCES + ["abi_cache.cpp", "cache_rows.hip", "cache_attention.hip"]

pytestmark = [pytest.mark.skipif(not os.path.exists(base.CLANG), reason="the ROCm clang is not installed"),
              pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake device pointers; run where no GPU is visible")]


def test_cache_abi_host_code_under_sanitizers(tmp_path):
    inc = ["-I", os.path.join(base.ROOT, "include"), "-I", os.path.join(base.ROCM, "include")]
    jobs = []
    for src in SOURCES:
        obj = str(tmp_path / (os.path.splitext(src)[0] + ".o"))
        jobs.append(([base.CLANG, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", *base.HOST_SAN, *inc,
                      "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-c", os.path.join(base.CSRC, src),
                      "-o", obj], obj))
    drv = str(tmp_path / "driver.o")
    jobs.append(([base.CLANG, "-x", "c++", "-O1", "-g", "-std=c++17", *base.SAN, *inc, "-D__HIP_PLATFORM_AMD__", "-c",
                  os.path.join(base.ROOT, "tests", "cache_abi_sanitize_driver.cpp"), "-o", drv], drv))
    with cf.ThreadPoolExecutor(max_workers=4) as ex:
        for (cmd, _), (rc, out) in zip(jobs, ex.map(lambda j: base._run(j[0]), jobs)):
            assert rc == 0, f"{' '.join(cmd)}\n{out}"
    exe = str(tmp_path / "cache_abi_driver")
    rc, out = base._run([base.CLANG, *base.SAN, *[o for _, o in jobs], "-L", os.path.join(base.ROCM, "lib"), "-lamdhip64",
                         f"-Wl,-rpath,{os.path.join(base.ROCM, 'lib')}", "-o", exe])
    assert rc == 0, out
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    rc, out = base._run([exe], env=env, timeout=300)
    print(out)
    assert rc == 0, out
    assert " 0 failures" in out, out
