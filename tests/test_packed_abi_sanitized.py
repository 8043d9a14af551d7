"""The host layers of packed rows and of the eviction under AddressSanitizer and UndefinedBehaviorSanitizer: tests/abi_host/packed_check.c
drives their entry points through their argument checks, every size and stride to the ends of its type, linked with the host
sources built by g++ under both sanitizers and with the kernel objects of the normal build.

Host only, where no GPU is present: a call that reaches a launch cannot touch a device."""
import os

import pytest

from tests.test_abi_sanitized import CSRC, ROCM, ROOT, SANITIZE, _skip_reason
from tests.test_cache_abi_sanitized import _run


@pytest.mark.skipif(_skip_reason() is not None, reason=str(_skip_reason()))
def test_packed_host_layers_under_sanitizers(tmp_path):
    from paper_2609_01925_amd import build as B
    hip, cpp = B.sources()
    kernels = [os.path.join(B.BUILD, f[:-4] + ".o") for f in hip]
    if not all(os.path.exists(f) for f in kernels):
        B.build()
    host = ["-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{B.INCLUDE}", f"-I{CSRC}"]
    objects = []
    for name in cpp:
        objects.append(str(tmp_path / (name[:-4] + ".o")))
        _run(["g++", "-std=c++17", "-fPIC", *SANITIZE, *host, "-c", os.path.join(CSRC, name), "-o", objects[-1]])
    objects.append(str(tmp_path / "packed_check.o"))
    _run(["gcc", "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", *SANITIZE, f"-I{B.INCLUDE}", "-c",
          os.path.join(ROOT, "tests", "abi_host", "packed_check.c"), "-o", objects[-1]])
    exe = str(tmp_path / "packed_check")
    _run(["g++", "-fsanitize=address,undefined", *objects, *kernels, f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib",
          "-lpthread", "-lm", "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    p = _run([exe], env=env, timeout=120)
    assert " 0 failures" in p.stdout and "runtime error" not in p.stderr and "AddressSanitizer" not in p.stderr, p.stdout + p.stderr
