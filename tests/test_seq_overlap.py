"""The test of shared memory, compiled by itself (CPU only)."""
import os
import subprocess

import pytest
from test_sanitizers import CLANG, ENV, HERE, OUT, ROOT, SAN


def test_rows_that_share_memory_are_found():
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ with sanitizer runtimes in this image")
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "seq_overlap")
    cmd = [CLANG, "-std=c++17", "-O1", "-I" + os.path.join(ROOT, "paper_2007_06000_amd", "csrc"), *SAN, os.path.join(HERE, "seq_overlap.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    r = subprocess.run([exe], capture_output=True, text=True, env=ENV, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "ERROR: AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, r.stderr[-4000:]
