"""CPU tests of the operators on paged caches at the ends of their arguments' ranges."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import pages as pg
from test_pages_host import LAY, L, append, attend, gather

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


def test_integers_of_more_than_32_bits_are_refused():
    pool, table = pg.new_pool(LAY, 2, device="cpu"), torch.zeros((1, 2), dtype=torch.int32)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    for bad in (2 ** 31, 2 ** 32 + 1, -2 ** 31 - 1, 2 ** 64):
        for name in ("layer", "window", "split_tokens", "sm_quota"):
            with pytest.raises(ValueError, match=name):
                pg.attend(LAY, pool, table, q, [1], [1], **{name: bad})
        for name in ("layer", "sm_quota"):
            with pytest.raises(ValueError, match=name):
                pg.append(LAY, pool, table, q, q, [1], [1], **{name: bad})
        with pytest.raises(ValueError, match="sm_quota"):
            pg.copy(LAY, pool, pool, ([0], [1]), sm_quota=bad)
        with pytest.raises(ValueError, match="sm_quota"):
            pg.gather(LAY, pool, table, [1], sm_quota=bad)
        for name in LAY._fields[:4]:
            with pytest.raises(ValueError, match=name):
                pg.new_pool(LAY._replace(**{name: bad}), 1, device="cpu")
        for args in ((bad, 32, 1), (1, bad, 1), (1, 32, bad)):
            with pytest.raises(ValueError):
                pg.Book(*args)
        book = pg.Book(4, 32, 2)
        book.extend([0], [40])
        assert book.len(bad) == -1
        for fn in (lambda: book.shorten([0], bad), lambda: book.extend([0], [bad]), lambda: book.fork([0], [bad])):
            with pytest.raises(ValueError):
                fn()
        assert book.used == 2 and book.len(0) == 40


def test_compaction_with_any_number_of_moves_at_most():
    for most, moves in ((2 ** 31 - 1, 2), (2 ** 32 + 1, 2), (2 ** 64, 2), (1, 1), (0, 0)):
        book = pg.Book(8, 32, 3)
        book.extend([0, 1], [64, 64])
        book.shorten([0], 0)
        assert [len(m) for m in book.compact(most)] == [moves] * 3
    for most in (-1, -2 ** 31, -2 ** 31 - 1, -2 ** 32):
        with pytest.raises(B.EbrlError):
            book.compact(most)


def test_planes_too_far_apart_are_refused():
    """The distance of planes travels as a number of rows in 32 bits."""
    assert pg._rows32([0, 2 ** 31 - 1]) == [0, 2 ** 31 - 1]
    with pytest.raises(ValueError):
        pg._rows32([5, 2 ** 31])


def test_scales_that_leave_fp32_are_refused():
    """The kernels take scores in units of log 2: scale * 1.4427 has to be a number."""
    for scale in (2.4e38, -2.4e38, 3.4e38):
        assert attend(scale=scale) == B.ERR_INVALID_ARG
    for scale in (2.3e38, -2.3e38, 1e-45, 0.0):
        assert attend(scale=scale) != B.ERR_INVALID_ARG
