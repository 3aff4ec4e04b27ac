"""CPU tests of the operators on paged caches at the ends of their arguments' ranges."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_token_ranges_do_not_wrap(tmp_path):
    exe = str(tmp_path / "pages_span_driver")
    cmd = ["g++", "-std=c++17", "-g", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "pages_span_sanitize_driver.cpp"), "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert b.returncode == 0, b.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "pages span driver: ok" in r.stdout, (r.stdout + r.stderr)[-4000:]
