"""Exact attention's host code (argument checks, bucket borders, launch rules) under AddressSanitizer and
UndefinedBehaviorSanitizer, built as test_abi_sanitized.py builds the rest (CPU only)."""
import os
import shutil
import subprocess

import pytest

from paper_2201_12854_amd import build_lib

HERE = os.path.dirname(os.path.abspath(__file__))


def test_exact_checks_under_host_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]

    def run(*cmd, **kw):
        r = subprocess.run(cmd, capture_output=True, text=True, **kw)
        assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
        return r.stdout + r.stderr

    objs = []
    for src in build_lib.SOURCES:
        built = os.path.join(build_lib.BUILD, src + ".o")
        if src.endswith(".cpp") or not os.path.exists(built):
            built = str(tmp_path / (src + ".o"))
            run(hipcc, *build_lib.CXXFLAGS, *(san if src.endswith(".cpp") else []), "-x", "hip", "-c",
                os.path.join(build_lib.CSRC, src), "-o", built)
        objs.append(built)
    drv, exe = str(tmp_path / "exact_checks.o"), str(tmp_path / "exact_checks")
    run(hipcc, *build_lib.CXXFLAGS, *san, "-I", os.path.join(build_lib.ROOT, "include"), "-x", "hip", "-c",
        os.path.join(HERE, "sanitize", "exact_checks.cpp"), "-o", drv)
    run(hipcc, f"--offload-arch={build_lib.ARCH}", *san, drv, *objs, "-o", exe)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", HIP_VISIBLE_DEVICES="")
    out = run(exe, env=env, timeout=120)
    assert "all exact checks passed" in out and "runtime error" not in out, out[-3000:]
