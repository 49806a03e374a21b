"""The upload staging (csrc/staging.h) on two devices that the host simulates, under the address and
undefined-behaviour sanitizers: tests/native/staging.cpp."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_uploads_to_two_devices(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    native, out = os.path.join(ROOT, "tests", "native"), str(tmp_path / "staging")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-I", os.path.join(native, "fake_hip"), "-I", os.path.join(ROOT, "paper_2601_11652_amd", "csrc"),
                        os.path.join(native, "staging.cpp"), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    # buffers and events live as long as their thread, as in the library
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0")
    r = subprocess.run([out], capture_output=True, text=True, timeout=60, env=env)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "staging ok" in r.stdout
