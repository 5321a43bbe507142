"""Host side of the operators around the training step (layer norm, AdamW, rotary positions with several axes) under
AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: checks, launch tables and frequencies, compiled from the library's
source by the host compiler and linked with recording stand-ins for the launchers (tests/host_sanitizer/train_ops_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HS = os.path.join(ROOT, "tests", "host_sanitizer")
CSRC = os.path.join(ROOT, "paper_2505_16710_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_entry_points_are_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "train_ops_run")
    flags = ["-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
             "-static-libasan", "-static-libubsan", "-Wall", "-I", HS, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    srcs = [os.path.join(CSRC, "train_ops_api.cpp"), os.path.join(HS, "train_ops_driver.cpp")]
    r = subprocess.run(["g++", *flags, *srcs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1"))
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    assert "all checks passed" in r.stdout


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_refused_calls_launch_nothing(tmp_path):
    """The layer norm's refusals at the library's own limits (tests/host_sanitizer/train_ops_refusals.cpp)."""
    exe = str(tmp_path / "refusals_run")
    flags = ["-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-static-libubsan",
             "-Wall", "-I", HS, "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    srcs = [os.path.join(CSRC, "train_ops_api.cpp"), os.path.join(HS, "train_ops_refusals.cpp")]
    r = subprocess.run(["g++", *flags, *srcs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "all checks passed" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
