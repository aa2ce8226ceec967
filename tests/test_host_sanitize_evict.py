"""The block allocator's evictions built with g++ under AddressSanitizer and
UndefinedBehaviorSanitizer and driven by random operations
(tests/sanitize/evict_fuzz.cpp).  CPU only: no HIP code is compiled."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_evictions_under_address_and_ub_sanitizers(tmp_path):
    exe = str(tmp_path / "evict_fuzz")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", os.path.join(HERE, "sanitize", "evict_fuzz.cpp"),
           os.path.join(ROOT, "paper_2609_37062_amd", "csrc", "alloc.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe, "200"], capture_output=True, text=True, timeout=600,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1"))
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    counts = [int(t) for t in r.stdout.replace(",", " ").split() if t.isdigit()]
    assert len(counts) == 4 and min(counts) > 0, r.stdout  # (every kind of call was reached)
