"""The book of a paged cache (host-only source) under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_book_is_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "pages_book_driver")
    cmd = ["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-x", "c++",
           os.path.join(ROOT, "paper_2609_27547_b200", "csrc", "pages_book.cu"), os.path.join(ROOT, "tests", "pages_book_sanitize_driver.cpp"), "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert b.returncode == 0, b.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "pages book driver: ok" in r.stdout, (r.stdout + r.stderr)[-4000:]
