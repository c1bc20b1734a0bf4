"""The host-only code of the transformer block's operators built on its own with AddressSanitizer and
UndefinedBehaviorSanitizer and driven by tests/c/block_host_checks.cpp, which also takes its memory away.  No GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_05588_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_block_host_code_under_asan_and_ubsan(tmp_path):
    exe = tmp_path / "block_host_checks"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-Wall",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", "/opt/rocm/include",
           os.path.join(CSRC, "daso_block_host.cpp"), os.path.join(CSRC, "daso_train_host.cpp"),
           os.path.join(ROOT, "tests", "c", "block_host_checks.cpp"), "-o", str(exe)]
    built = subprocess.run(cmd, capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert res.returncode == 0, res.stderr[-4000:]
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, res.stderr[-4000:]
    assert "block host checks ok" in res.stdout


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_accepted_rows_touch_no_other_rows(tmp_path):
    exe = tmp_path / "block_alias_checks"
    cmd = ["g++", "-std=c++17", "-O2", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           "-I", "/opt/rocm/include", os.path.join(CSRC, "daso_block_host.cpp"), os.path.join(CSRC, "daso_train_host.cpp"),
           os.path.join(ROOT, "tests", "c", "block_alias_checks.cpp"), "-o", str(exe)]
    built = subprocess.run(cmd, capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-4000:]
    res = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-4000:]
    assert "block alias checks ok" in res.stdout
