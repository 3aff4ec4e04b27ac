"""GPU tests of the operators on paged caches at the ends of their arguments' ranges.  References and tolerances are those of test_pages_gpu.py."""
import math

import pytest
import torch

from paper_2609_27547_b200 import binding as B
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


def constant(lay, n, key, value, seed=0):
    """One sequence whose keys are key[t] along the first column and 0 elsewhere, and whose values are value[t] in all columns."""
    cache = Cache(lay, [n], seed=seed)
    kv = torch.zeros((1, 2, lay.n_kv_heads, n, lay.head_dim))
    kv[0, 0, :, :, 0] = key
    kv[0, 1] = value[:, None]
    kv = kv.to(lay.dtype)
    cache.kv = [kv.double()]
    elems, _ = pg.views(lay, cache.pool)
    T = lay.page_tokens
    for j, p in enumerate(cache.rows[0]):
        k = min(T, n - j * T)
        elems[p, 0, :, :, :k] = kv[0, :, :, j * T:j * T + k].cuda()
    return cache


@pytest.mark.parametrize("hd,m", [(128, 200), (128, 100), (64, 100), (32, 100)])
def test_sums_of_large_values_stay_finite(hd, m):
    """A first tile far below the others, just so much that no single tile's weights (2^8.93 each) ask for another reference: what they add up to is
    bounded all the same.  Sums may be 2^16 times the values: 4e33 * 2^16 = 2.6e38 is finite, 2^16 times 130 tiles would not be."""
    lay = pg.Layout(1, 1, hd, 128, BF)
    n = 130 * 128
    key = torch.full((n,), 6.1875)
    key[:128] = 0
    g = torch.Generator().manual_seed(hd)
    cache = constant(lay, n, key, 4e33 * (0.5 + 0.5 * torch.rand(n, generator=g)))
    q = torch.zeros((m, 1, hd), dtype=BF, device="cuda")
    q[:, 0, 0] = 1
    for split in (-1, 1024):
        out, lse = pg.attend(lay, cache.pool, cache.table, q, [m], [n], scale=1.0, causal=False, split_tokens=split)
        check(cache, 0, q, [m], out, lse, scale=1.0, causal=False)


@pytest.mark.parametrize("hd", [128, 64])
def test_many_tokens_of_one_weight(hd):
    """More tokens than the bound of the sums: the reference leaves the largest score behind.  No reference does so with a subnormal scale: sums are then as large as the
    number of tokens, 2e5 * 1.5e33 = 3e38 at most."""
    lay = pg.Layout(1, 1, hd, 256, BF)
    n, m = 200_000, 130
    g = torch.Generator().manual_seed(hd)
    value = 0.5 + 0.5 * torch.rand(n, generator=g)
    q = torch.ones((m, 1, hd), dtype=BF, device="cuda")
    for scale, size in ((0.125, 4e33), (1e38, 4e33), (1e-40, 1.5e33)):
        cache = constant(lay, n, torch.zeros(n), size * value)
        out, lse = pg.attend(lay, cache.pool, cache.table, q, [m], [n], scale=scale, causal=False, split_tokens=-1)
        check(cache, 0, q, [m], out, lse, scale=scale, causal=False)


@pytest.mark.parametrize("hd,m", [(128, 200), (128, 20), (64, 40), (32, 40)])
def test_what_a_wait_that_ran_out_left_unfinished_is_not_joined(hd, m):
    """Cut sequences whose pieces never came to an end leave out and lse as they are; the queries, too, where out is q."""
    lay = pg.Layout(1, 2, hd, 64, BF)
    lens, counts = [300, 100, 700], [m, m, m]
    cache = Cache(lay, lens, seed=1)
    q = queries(lay, 3 * m, 1)
    L = pg._load()
    pg.check()
    for same in (False, True):
        out = q.clone() if same else torch.full_like(q, 7.0)
        lse = torch.full((3 * m, 2), 7.0, device="cuda")
        L.ebrl_pages_test_drop_copies(20_000_000)
        try:
            pg.attend(lay, cache.pool, cache.table, out if same else q, counts, lens, out=out, lse=lse, split_tokens=128)
        finally:
            L.ebrl_pages_test_drop_copies(0)
        with pytest.raises(B.EbrlError) as e:
            pg.check()
        assert e.value.status == B.ERR_TIMEOUT
        assert torch.equal(out, q) if same else bool((out == 7).all())
        assert bool((lse == 7).all())
    out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, lens, split_tokens=128)
    check(cache, 0, q, counts, out, lse)
    pg.check()


@pytest.mark.parametrize("dtype", [BF, F])
def test_a_group_that_was_reset_as_a_whole(dtype):
    """The book's table of sequences without tokens has no columns; every operator takes it."""
    lay = pg.Layout(1, 2, 64, 32, dtype)
    book, pool = pg.Book(8, 32, 3), pg.new_pool(lay, 8)
    table = book.table([0, 1, 2], device="cuda")
    assert table.shape == (3, 0)
    before = pool.clone()
    x = queries(lay, 60, 1)
    pg.append(lay, pool, table, x[:0], x[:0], [0, 0, 0], [0, 0, 0])
    for counts in ([0, 0, 0], [1, 0, 2], [3, 50, 1]):
        q = x[:sum(counts)]
        for causal in (True, False):
            out, lse = pg.attend(lay, pool, table, q, counts, [0, 0, 0], causal=causal)
            assert out.shape == q.shape and bool((out == 0).all()) and bool((lse == -math.inf).all())
    planes = pg.gather(lay, pool, table, [0, 0, 0])
    assert [tuple(p.shape) for p in planes] == [(1, 2, 0, 128)] * 3
    whole = torch.full((3, 1, 2, 5, 128), 7.0, dtype=dtype, device="cuda")
    pg.gather(lay, pool, table, [0, 0, 0], whole)
    assert bool((whole == 7).all()) and torch.equal(pool, before)


def test_a_sequence_with_too_many_items_is_refused_before_anything_is_enqueued():
    """1024 sequences that fill a launch, and one whose query rows and heads make 2^31 items."""
    lay = pg.Layout(1, 64, 32, 32, F)
    n, m, huge = 1025, 17, 2 ** 30 - 1
    cache = Cache(lay, [2], seed=1)
    table = cache.table[:1, :1].expand(n, 1).contiguous()
    q = queries(lay, 1, 1)
    out = torch.full(((n - 1) * m, 64, 32), 7.0, device="cuda")
    counts, lens = [m] * (n - 1) + [huge], [2] * (n - 1) + [1]
    L, ints = pg._load(), lambda v: (pg.C.c_int32 * len(v))(*v)
    st = L.ebrl_pages_attend(pg._pool(lay, cache.pool), cache.pool.data_ptr(), cache.n_pages, n, table.data_ptr(), 1, ints(counts), ints(lens), 0, q.data_ptr(), 0, 64,
                             out.data_ptr(), 64 * 32, None, 1.0, 0, 0, -1, None, 0, 0, torch.cuda.current_stream().cuda_stream)
    assert st == B.ERR_UNSUPPORTED and bool((out == 7).all())
    L.ebrl_pages_attend(pg._pool(lay, cache.pool), cache.pool.data_ptr(), cache.n_pages, n - 1, table.data_ptr(), 1, ints(counts), ints(lens), 0, q.data_ptr(), 0, 64,
                        out.data_ptr(), 64 * 32, None, 1.0, 0, 0, -1, None, 0, 0, torch.cuda.current_stream().cuda_stream)
    assert bool((out[::m] == out[0]).all()) and not bool((out == 7).any())


@pytest.mark.parametrize("hd", [128, 64, 32])
def test_scales_that_are_not_positive_with_many_rows(hd):
    """bf16 rows that a positive scale would send to the tensor-memory kernel."""
    lay = pg.Layout(1, 2, hd, 64, BF)
    lens, counts = [700, 90, 40, 1300], [33, 90, 50, 1]
    cache = Cache(lay, lens, hide=0.2, lost=0.1, seed=hd)
    for G in (1, 3):
        q = queries(lay, sum(counts), G, seed=G)
        for scale in (0.0, -0.1):
            for kw in (dict(), dict(split_tokens=-1), dict(split_tokens=256), dict(sm_quota=20), dict(window=37), dict(causal=False)):
                out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, lens, scale=scale, **kw)
                check(cache, 0, q, counts, out, lse, scale=scale, causal=kw.get("causal", True), window=kw.get("window", 0))


@pytest.mark.parametrize("dtype,hd,m", [(BF, 64, 1), (BF, 128, 1), (BF, 64, 20), (BF, 128, 20), (BF, 128, 200), (BF, 64, 40), (BF, 32, 40), (F, 64, 1), (F, 64, 40), (F, 128, 20)])
def test_scores_whose_last_bits_are_large(dtype, hd, m):
    """Scores of one size, however large, are equal weights.  lse: the score is one product, with two constants (log2 e, ln 2) and three roundings around it, each off
    by 2^-24 of it at most, together less than 2^-21; fp32 operands lose 5 * 2^-22 besides."""
    lay = pg.Layout(1, 1, hd, 64, dtype)
    n = 300
    g = torch.Generator().manual_seed(hd)
    lose = 2.0 ** -21 + (5 * 2.0 ** -22 if dtype is F else 0)
    for size in (1e4, 1e7, 1e9, 1e10, 1e12, 1e20, 1e30, 1e38):
        for sign in (1, -1):
            cache = constant(lay, n, torch.full((n,), math.sqrt(size)), 0.5 + torch.rand(n, generator=g))
            q = torch.zeros((m, 1, hd), dtype=dtype, device="cuda")
            q[:, :, 0] = sign * math.sqrt(size)
            score = float(q[0, 0, 0].double() * cache.kv[0][0, 0, 0, 0, 0])
            for split in (0, -1, 128):
                out, lse = pg.attend(lay, cache.pool, cache.table, q, [m], [n], scale=1.0, split_tokens=split)
                alike = torch.log(torch.arange(n - m + 1, n + 1, device="cuda", dtype=torch.float64))[:, None]
                check(cache, 0, torch.zeros_like(q), [m], out, alike.float(), scale=1.0)
                assert bool(((lse.double() - alike - score).abs() <= lose * (abs(score) + alike)).all()), (size, sign, split)


def test_one_visible_token_with_any_score():
    """Its values are the result: off by the rounding of its weight (2^-8; the weight is 2 to the power of what the reference lost when it was rounded, which is not
    always a bf16 number, while the sum that divides it is not rounded) and by that of the result (2^-8), together (1 + 2^-8)^2 - 1 = 2^-7 + 2^-16 of them at most."""
    lay = pg.Layout(1, 1, 64, 64, BF)
    cache = Cache(lay, [200], seed=3)
    _, words = pg.views(lay, cache.pool)
    words.zero_()
    words[cache.rows[0][1], 0] = 1 << 5                  # token 69
    want = cache.kv[0][0, 1, 0, 69].to(BF).cuda()
    for m in (1, 20, 100):
        for size in (1.0, 1e5, 1e8, 1e15):
            q = (queries(lay, m, 1).float() * size).to(BF)
            out, lse = pg.attend(lay, cache.pool, cache.table, q, [m], [200], causal=False)
            assert bool(((out.double() - want.double()).abs() <= (2.0 ** -7 + 2.0 ** -16) * want.double().abs()).all()) and bool(torch.isfinite(lse).all())
