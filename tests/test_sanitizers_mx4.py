"""Sanitizer build of the argument validation of the products in 4 bits and of the heads'
norms (CPU only): tcu_mx4_abi.cpp, tcu_heads_abi.cpp and tcu_abi.cpp as host code with
AddressSanitizer and UndefinedBehaviorSanitizer, driven by tests/sanitize/mx4_driver.c."""
import os
import shutil

import pytest
import torch

checks = pytest.importorskip("test_sanitizers")
KERNEL_OBJS = checks.KERNEL_OBJS + ["tcu_mx4.o", "tcu_mx4_gemm.o", "tcu_heads.o"]


@pytest.mark.skipif(shutil.which("g++") is None or torch.cuda.is_available(),
                    reason="needs g++ and a machine without a GPU (valid calls must stop at the "
                           "device query)")
def test_validation_under_asan_ubsan(tmp_path):
    objects = [os.path.join(checks.ROOT, "_build", o) for o in KERNEL_OBJS]
    if not all(os.path.exists(o) for o in objects):
        from paper_1908_06649_amd import build as hip_build
        hip_build.build()
    source = os.path.join(checks.ROOT, "paper_1908_06649_amd", "csrc")
    inc = ["-I" + os.path.join(checks.ROOT, "include"), "-I" + source]
    host = []
    for name in ("tcu_abi", "tcu_mx4_abi", "tcu_heads_abi"):
        host.append(str(tmp_path / (name + ".o")))
        checks._run(["g++", "-std=c++17", *checks.SAN, "-D__HIP_PLATFORM_AMD__",
                     f"-I{checks.ROCM}/include", *inc, "-c", os.path.join(source, name + ".cpp"),
                     "-o", host[-1]])
    driver, exe = str(tmp_path / "driver.o"), str(tmp_path / "mx4_driver")
    checks._run(["gcc", "-std=c11", *checks.SAN, *inc, "-c",
                 os.path.join(checks.HERE, "mx4_driver.c"), "-o", driver])
    checks._run(["g++", *checks.SAN, driver, *host, *objects, f"-L{checks.ROCM}/lib",
                 "-lamdhip64", f"-Wl,-rpath,{checks.ROCM}/lib", "-o", exe])
    assert "0 failures" in checks._run([exe], env=checks._env(leaks=False)).stdout
