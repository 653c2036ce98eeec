"""The host code of the operators on paged caches under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): ``abi_cache.cpp`` and what it shares with
``abi.cpp`` and ``planner.cpp``, with launchers that report
hipErrorNotSupported, run by the host tests through ``MSTAR_ATTN_LIB``."""
import os
import subprocess
import sys

from tests.test_host_sanitizers import CSRC, ENV, FLAGS, ROOT, SAN, _build, _gxx


def test_host_tests_against_the_sanitized_library(tmp_path):
    gxx, asan = _gxx()
    lib = str(tmp_path / "libmstar_attn_sanitized.so")
    _build([gxx, *FLAGS, "-fPIC", "-shared", *(os.path.join(CSRC, f) for f in ("abi.cpp", "abi_cache.cpp", "planner.cpp")),
            os.path.join(SAN, "kernels_stub.cpp"), os.path.join(SAN, "cache_stub.cpp"), "-L/opt/rocm/lib",
            "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", lib])
    env = {**os.environ, **ENV, "MSTAR_ATTN_LIB": lib, "LD_PRELOAD": asan}
    res = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu",
                          os.path.join(ROOT, "tests", "test_cache_host.py")],
                         capture_output=True, text=True, env=env, cwd=ROOT, timeout=900)
    print(res.stdout[-3000:] + res.stderr[-4000:])
    assert res.returncode == 0
    assert "Sanitizer" not in res.stderr and "runtime error" not in res.stderr
    assert " passed" in res.stdout and "failed" not in res.stdout
