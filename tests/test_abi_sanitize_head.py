"""The language-model head's entry points under AddressSanitizer and UndefinedBehaviorSanitizer on the host side (CPU
only): the objects of test_abi_sanitize's build, linked with a driver of their own."""
import os
import subprocess

import pytest
import test_abi_sanitize as base

DRIVER = os.path.join(base.ROOT, "tests", "abi_validate_head.cpp")


@pytest.mark.skipif(not (os.path.exists(base.HIPCC) and os.path.exists(base.CLANG)), reason="ROCm compilers not found")
def test_head_host_side_under_sanitizers(tmp_path):
    base._build()
    objs = [os.path.join(base.OUT, os.path.basename(s) + ".o") for s in base._sources()]
    san = "-fsanitize=" + ",".join(base.SAN)
    exe, drv = str(tmp_path / "abi_validate_head"), str(tmp_path / "abi_validate_head.o")
    for cmd in ([base.CLANG, "-O1", "-g", "-std=c++17", "-I", base.INCLUDE, "-D__HIP_PLATFORM_AMD__", "-I",
                 "/opt/rocm/include", san, "-c", DRIVER, "-o", drv],
                [base.CLANG, san, drv, *objs, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-2000:] + r.stderr[-4000:]
