"""The argument checks of ditupdate.h and ditint8.h built with g++ under AddressSanitizer and UndefinedBehaviorSanitizer, driven by
tests/host_sanitize/update_driver.cpp. No GPU; the device code is not compiled for it."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_19004_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_update_checks_under_asan_ubsan(tmp_path):
    exe = str(tmp_path / "update_sanitize")
    b = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                        os.path.join(ROOT, "tests", "host_sanitize", "update_driver.cpp"), os.path.join(CSRC, "update_checks.cpp"),
                        os.path.join(CSRC, "host_checks.cpp"), "-o", exe], capture_output=True, text=True)
    assert b.returncode == 0, b.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout
