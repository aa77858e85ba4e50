"""Which layouts of a cache the append takes, on the CPU: tests/sanitize/append_layouts_check.cpp
builds generation.cpp under AddressSanitizer and UndefinedBehaviorSanitizer with stand-ins for its
launches and compares small layouts of keys and values vector by vector."""
import os
import shutil
import subprocess
import sys
from pathlib import Path

import pytest

HERE = Path(__file__).resolve().parent


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_layouts(tmp_path):
    sys.path.insert(0, str(HERE / "sanitize"))
    try:
        import build as san_build
    finally:
        sys.path.pop(0)
    exe = tmp_path / "append_layouts_check"
    subprocess.run(["g++", "-std=c++17", *san_build.SAN, *san_build.INC, "-Wall", "-Wextra",
                    str(san_build.CSRC / "generation.cpp"), str(HERE / "sanitize" / "append_layouts_check.cpp"),
                    "-o", str(exe)], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout, r.stderr[-4000:])
    assert r.returncode == 0 and "runtime error" not in r.stderr and " 0 failed" in r.stdout
