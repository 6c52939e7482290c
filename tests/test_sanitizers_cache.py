"""The host side of the paged cache and of beams under AddressSanitizer + UndefinedBehaviorSanitizer: their ABI tests against the library whose
host code is instrumented, in a child process (see test_sanitizers.py).  No GPU is used."""
import glob
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_cache_and_beams_abi_under_host_sanitizers():
    sys.path.insert(0, ROOT)
    from paper_2605_08840_amd import build as hip_build
    rt = hip_build.asan_runtime()
    if not rt:
        pytest.skip("the toolchain ships no shared AddressSanitizer runtime")
    lib = hip_build.LIB_SAN
    newest = max(os.path.getmtime(x) for x in glob.glob(os.path.join(hip_build.CSRC, "*")) + glob.glob(os.path.join(ROOT, "include", "*.h")))
    if not os.path.exists(lib) or os.path.getmtime(lib) <= newest:
        lib = hip_build.build(verbose=False, sanitize=True)
    env = dict(os.environ)
    env["LD_PRELOAD"] = rt + (":" + env["LD_PRELOAD"] if env.get("LD_PRELOAD") else "")
    env["ASAN_OPTIONS"] = "detect_leaks=0:halt_on_error=1:abort_on_error=0"
    env["UBSAN_OPTIONS"] = "halt_on_error=1:print_stacktrace=1"
    env["RESTKV_LIB"] = lib
    # (-s: what a sanitizer prints before it ends the process is not held back)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-s", "-p", "no:cacheprovider",
           *(os.path.join(ROOT, "tests", f"test_{x}.py") for x in ("pages_abi", "beams_abi", "beams_list"))]
    r = subprocess.run(cmd, cwd=ROOT, env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, timeout=900)
    out = r.stdout.decode(errors="replace")
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[out.find("runtime error:") - 200:][:2000]
    assert r.returncode == 0 and " passed" in out, out[-4000:]
