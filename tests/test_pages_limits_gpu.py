"""GPU tests of the operators on paged caches at the ends of their arguments' ranges.  References and tolerances are those of test_pages_gpu.py."""
import pytest
import torch

from paper_2609_27547_b200 import pages as pg
from test_pages_gpu import BF, F, Cache, check, queries

pytestmark = pytest.mark.gpu

LARGEST = 2 ** 31 - 1

# (dtype, head_dim, query heads per key/value head): with 14 queries a call takes each of the kernels, with 16, 32, 128 and 256 rows an item
FORMS = [(BF, 64, 1), (BF, 64, 2), (BF, 64, 8), (BF, 32, 4), (BF, 128, 1), (BF, 128, 4), (BF, 128, 16), (F, 64, 1), (F, 128, 4), (F, 32, 8)]


@pytest.mark.parametrize("dtype,hd,G", FORMS)
def test_windows_and_pieces_that_end_nothing(dtype, hd, G):
    """More queries than tokens, so that some stand before the first one, with a window and pieces as large as the types allow."""
    lay = pg.Layout(1, 2, hd, 32, dtype)
    lens, counts = [10, 0, 6, 200], [14, 5, 14, 14]
    cache = Cache(lay, lens, seed=hd + G)
    q = queries(lay, sum(counts), G, seed=G)
    want, want_l = pg.attend(lay, cache.pool, cache.table, q, counts, lens, split_tokens=-1)
    check(cache, 0, q, counts, want, want_l)
    for window in (200, LARGEST - 1, LARGEST):
        for split in (0, -1, 128, LARGEST // 128 * 128):
            out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, lens, window=window, split_tokens=split)
            check(cache, 0, q, counts, out, lse, window=window)
            if split < 0 or split > 200:
                assert torch.equal(out, want) and torch.equal(lse, want_l)


@pytest.mark.parametrize("dtype,hd,G", FORMS)
def test_the_largest_pieces_behind_a_window(dtype, hd, G):
    lay = pg.Layout(1, 2, hd, 64, dtype)
    lens, counts = [1000, 300], [14, 14]
    cache = Cache(lay, lens, seed=hd)
    q = queries(lay, sum(counts), G, seed=G)
    want = pg.attend(lay, cache.pool, cache.table, q, counts, lens, window=10, split_tokens=-1)
    check(cache, 0, q, counts, *want, window=10)
    for split in (1024, 2 ** 30, LARGEST // 128 * 128):
        got = pg.attend(lay, cache.pool, cache.table, q, counts, lens, window=10, split_tokens=split)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
