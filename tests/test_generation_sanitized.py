"""The host code of the C entry points of generation (generation.cpp,
nf4_linear_launch.hpp) under AddressSanitizer and UndefinedBehaviorSanitizer, on
the CPU: tests/sanitize/generation_host_check.cpp takes every argument of every
entry point through its ordinary values and the ends of its type, one and two at a
time, and stands in for the launches, checking what they are handed."""
import os
import shutil
import subprocess
import sys
from pathlib import Path

import pytest

HERE = Path(__file__).resolve().parent


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_generation_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    sys.path.insert(0, str(HERE / "sanitize"))
    try:
        import build as san_build
    finally:
        sys.path.pop(0)
    exe = tmp_path / "generation_host_check"
    subprocess.run(["g++", "-std=c++17", *san_build.SAN, *san_build.INC, "-Wall", "-Wextra",
                    str(san_build.CSRC / "generation.cpp"), str(HERE / "sanitize" / "generation_host_check.cpp"),
                    "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1:detect_stack_use_after_return=1:"
                                        "verify_asan_link_order=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout, r.stderr[-4000:])
    assert r.returncode == 0
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr
    assert " 0 failed" in r.stdout
