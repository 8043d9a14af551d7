"""The K/V cache's host layer under AddressSanitizer and UndefinedBehaviorSanitizer: tests/abi_host/cache_check.c
drives its entry points through their argument checks, every size and stride to the ends of its type, linked with
api.cpp and cache_api.cpp built by g++ under both sanitizers and with the kernel objects of the normal build.

Host only, where no GPU is present: a call that reaches a launch cannot touch a device."""
import os
import subprocess

import pytest

from tests.test_abi_sanitized import CSRC, ROCM, ROOT, SANITIZE, _skip_reason


@pytest.mark.skipif(_skip_reason() is not None, reason=str(_skip_reason()))
def test_cache_host_layer_under_sanitizers(tmp_path):
    from paper_2609_01925_amd import build as B
    kernels = [os.path.join(B.BUILD, f) for f in ("estimate.o", "select.o", "attn.o", "cache.o", "cache_attn.o", "pool.o")]
    if not all(os.path.exists(f) for f in kernels):
        B.build()
    host = ["-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{B.INCLUDE}", f"-I{CSRC}"]
    objects = []
    for name in ("api", "cache_api"):
        objects.append(str(tmp_path / f"{name}.o"))
        _run(["g++", "-std=c++17", "-fPIC", *SANITIZE, *host, "-c", os.path.join(CSRC, f"{name}.cpp"), "-o", objects[-1]])
    objects.append(str(tmp_path / "cache_check.o"))
    _run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", *SANITIZE, f"-I{B.INCLUDE}", "-c",
          os.path.join(ROOT, "tests", "abi_host", "cache_check.c"), "-o", objects[-1]])
    exe = str(tmp_path / "cache_check")
    _run(["g++", "-fsanitize=address,undefined", *objects, *kernels, f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib",
          "-lpthread", "-lm", "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    p = _run([exe], env=env, timeout=120)
    assert " 0 failures" in p.stdout and "runtime error" not in p.stderr and "AddressSanitizer" not in p.stderr, p.stdout + p.stderr


def _run(cmd, **kw):
    p = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert p.returncode == 0, f"$ {' '.join(cmd)}\n{p.stdout}\n{p.stderr}"
    return p
