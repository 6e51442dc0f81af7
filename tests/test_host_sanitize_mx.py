"""The host side of coded caches, reads and log probabilities under AddressSanitizer,
LeakSanitizer and UBSan, on the CPU: the sanitized library of test_host_sanitize with a driver
of its own (tests/host/mx_checks.cpp)."""
import os
import shutil
import subprocess

import pytest

import test_host_sanitize as H
from paper_2609_37029_amd import build as B


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc is required to build the sanitized library")
def test_mx_host_under_asan_and_ubsan(tmp_path):
    H._build()
    objs = [os.path.join(H.OUT, os.path.splitext(s)[0] + ".o") for s in B.SOURCES]
    exe = str(tmp_path / "mx_checks")
    r = subprocess.run([H.CLANG, "-O1", "-std=c++17", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", "-g",
                        "-I", os.path.join(H.ROOT, "include"),
                        os.path.join(H.HOST, "mx_checks.cpp"), "-o", exe] + objs +
                       ["-L", H.ROCM_LIB, "-lamdhip64", "-Wl,-rpath," + H.ROCM_LIB],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, HIP_VISIBLE_DEVICES="",
               ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-6000:])
    assert "mx checks ok" in r.stdout
