"""CPU tests of the operators on paged caches at the ends of their arguments' ranges."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import pages as pg
from test_pages_host import L, append, attend, gather

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_token_ranges_do_not_wrap(tmp_path):
    exe = str(tmp_path / "pages_span_driver")
    cmd = ["g++", "-std=c++17", "-g", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "pages_span_sanitize_driver.cpp"), "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert b.returncode == 0, b.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "pages span driver: ok" in r.stdout, (r.stdout + r.stderr)[-4000:]


def test_sequences_without_tokens_need_no_table():
    no = dict(table=None, ts=0, len=[0, 0, 0])
    assert append(new=[0, 0, 0], **no) == B.OK
    assert attend(new=[0, 0, 0], **no) == B.OK
    for fn in (lambda: attend(new=[2, 0, 1], **no), lambda: gather(planes=[0, 0, 0], **no)):
        st = fn()
        assert st != B.ERR_INVALID_ARG, L.ebrl_pages_last_error()
        assert st == B.ERR_CUDA or torch.cuda.is_available()
    for op in (append, attend, gather):      # one with tokens does
        assert op(table=None) == B.ERR_INVALID_ARG


def test_table_of_empty_sequences():
    book = pg.Book(4, 32, 3)
    book.extend([1], [33])
    assert book.table([0, 2]).shape == (2, 0) and book.table([0, 2], 2).tolist() == [[-1, -1]] * 2
    assert book.table([0, 1]).tolist() == [[-1, -1], [0, 1]]
    with pytest.raises(B.EbrlError):
        book.table([0, 1], 0)
    seqs = (pg.C.c_int32 * 1)(0)
    assert L.ebrl_pages_book_table(book._b, 1, seqs, None, 0) == B.OK
    for stride in (1, -1):
        assert L.ebrl_pages_book_table(book._b, 1, seqs, None, stride) == B.ERR_INVALID_ARG
