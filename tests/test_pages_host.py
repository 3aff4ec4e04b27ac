"""CPU-only tests of the operators on paged caches: the page's layout, every refusal (arguments are checked before anything
touches a device), and the book against a model in Python."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import pages as pg

L = pg._load()
LAY = pg.Layout(2, 4, 64, 32, torch.bfloat16)
P0 = 0x10000     # an aligned address that is never touched


def lay(dtype=B.BF16, **kw):
    return C.byref(pg._CLayout(*LAY._replace(**kw)[:4], dtype))


def ints(v):
    return None if v is None else (C.c_int32 * max(1, len(v)))(*v)


def ptrs(v):
    return None if v is None else (C.c_void_p * max(1, len(v)))(*v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_page_layout(dtype):
    for l in (LAY, pg.Layout(1, 1, 32, 32), pg.Layout(3, 2, 128, 256), pg.Layout(1, 16, 128, 64)):
        l = l._replace(dtype=dtype)
        n = l.kv_layers * 2 * l.n_kv_heads * l.page_tokens * l.head_dim * dtype.itemsize
        assert l.page_bytes == -(-(n + l.page_tokens // 8) // 128) * 128
        pool = pg.new_pool(l, 3, device="cpu")
        elems, words = pg.views(l, pool)
        assert elems.shape == (3, l.kv_layers, 2, l.n_kv_heads, l.page_tokens, l.head_dim) and words.shape == (3, l.page_tokens // 32)
        elems[2, -1, 1, -1, -1, -1] = 1.5
        words[2, -1] = 9
        at = pool[2]
        assert at[n - dtype.itemsize:n].view(dtype).item() == 1.5
        assert at[n:n + l.page_tokens // 8].view(torch.int32)[-1].item() == 9


@pytest.mark.parametrize("kw", [dict(kv_layers=0), dict(n_kv_heads=0), dict(head_dim=48), dict(head_dim=256), dict(page_tokens=0), dict(page_tokens=16),
                                dict(page_tokens=48), dict(page_tokens=512), dict(kv_layers=5000), dict(n_kv_heads=5000), dict(dtype=B.E4M3), dict(dtype=7)])
def test_layouts_that_are_refused(kw):
    assert L.ebrl_pages_page_bytes(lay(**kw)) == 0
    assert len(L.ebrl_pages_last_error()) > 0
    if "dtype" not in kw:
        with pytest.raises(B.EbrlError):
            pg.new_pool(LAY._replace(**kw), 2, device="cpu")


def append(**kw):
    a = dict(lay=lay(), pool=P0, np=9, n=3, table=P0, ts=4, new=[1, 30, 0], len=[1, 100, 7], layer=1, k=P0, ks=256, v=P0, vs=768, mask=None, quota=0)
    a.update(kw)
    return L.ebrl_pages_append(a["lay"], a["pool"], a["np"], a["n"], a["table"], a["ts"], ints(a["new"]), ints(a["len"]), a["layer"], a["k"], a["ks"], a["v"],
                               a["vs"], a["mask"], a["quota"], None)


def attend(**kw):
    a = dict(lay=lay(), pool=P0, np=9, n=3, table=P0, ts=4, new=[1, 30, 0], len=[1, 100, 7], layer=1, q=P0, qs=512, heads=8, out=P0 + 65536, os=512, lse=P0,
             scale=0.125, causal=1, window=0, split=-1, ws=None, wsb=0, quota=0)
    a.update(kw)
    return L.ebrl_pages_attend(a["lay"], a["pool"], a["np"], a["n"], a["table"], a["ts"], ints(a["new"]), ints(a["len"]), a["layer"], a["q"], a["qs"], a["heads"],
                               a["out"], a["os"], a["lse"], a["scale"], a["causal"], a["window"], a["split"], a["ws"], a["wsb"], a["quota"], None)


def copy(**kw):
    a = dict(lay=lay(), pool=P0, np=9, dst=P0, dn=9, n=2, frm=[1, 1], to=[2, 3], tokens=None, quota=0)
    a.update(kw)
    return L.ebrl_pages_copy(a["lay"], a["pool"], a["np"], a["dst"], a["dn"], a["n"], ints(a["frm"]), ints(a["to"]), ints(a["tokens"]), a["quota"], None)


def gather(**kw):
    a = dict(lay=lay(), pool=P0, np=9, n=3, table=P0, ts=4, len=[1, 100, 0], planes=[P0, P0, 0], rows=None, rs=0, mask=None, quota=0)
    a.update(kw)
    return L.ebrl_pages_gather(a["lay"], a["pool"], a["np"], a["n"], a["table"], a["ts"], ints(a["len"]), ptrs(a["planes"]), ints(a["rows"]), a["rs"],
                               ptrs(a["mask"]), a["quota"], None)


CALLS = {"append": append, "attend": attend, "copy": copy, "gather": gather}
COMMON = [dict(lay=None), dict(n=-1), dict(np=-1), dict(np=0), dict(pool=None), dict(pool=P0 + 8)]
SEQS = [dict(len=None), dict(table=None), dict(table=P0 + 2), dict(ts=-1), dict(ts=3), dict(len=[1, -1, 7]), dict(len=[1, 129, 7])]
REFUSED = {
    "append": SEQS + [dict(layer=2), dict(layer=-1), dict(new=None), dict(new=[2, 30, 0]), dict(new=[1, -1, 0]), dict(k=None), dict(v=None), dict(k=P0 + 2), dict(v=P0 + 8),
                      dict(ks=-256), dict(vs=-8), dict(ks=252), dict(vs=260)],
    "attend": SEQS + [dict(layer=2), dict(layer=-1), dict(new=None), dict(new=[1, -1, 0]), dict(q=None), dict(q=P0 + 2), dict(heads=6), dict(heads=0), dict(heads=-4),
                      dict(qs=-512), dict(qs=508), dict(out=None), dict(out=P0 + 4), dict(os=508), dict(os=256), dict(out=P0, os=1024), dict(lse=P0 + 2), dict(scale=float("inf")),
                      dict(scale=float("nan")), dict(window=-1), dict(window=5, causal=0), dict(split=-2), dict(split=100)],
    "copy": [dict(dst=None), dict(dst=P0 + 8), dict(dst=P0 + 128), dict(dn=0), dict(frm=None), dict(to=None), dict(frm=[1, 9]), dict(frm=[-1, 1]), dict(to=[2, 9]), dict(to=[-1, 2]),
             dict(to=[2, 2]), dict(to=[1, 2]), dict(frm=[1, 2], to=[4, 1]), dict(tokens=[1, 33]), dict(tokens=[-1, 1])],
    "gather": SEQS + [dict(planes=None), dict(planes=[P0, 0, 0]), dict(planes=[P0 + 8, P0, 0]), dict(rows=[1, 99, 0]), dict(rs=255), dict(rs=260), dict(rs=-256)],
}


@pytest.mark.parametrize("op", list(CALLS))
def test_invalid_arguments_are_refused_before_the_device(op):
    for kw in COMMON + REFUSED[op]:
        st = CALLS[op](**kw)
        assert st == B.ERR_INVALID_ARG, (op, kw, st)
        assert len(L.ebrl_pages_last_error()) > 0
    assert CALLS[op](quota=-1) == B.ERR_QUOTA
    assert CALLS[op](lay=lay(head_dim=96)) == B.ERR_UNSUPPORTED
    assert CALLS[op](lay=lay(page_tokens=16)) == B.ERR_UNSUPPORTED
    assert CALLS[op](n=0) == B.OK                      # nothing to do, whatever else is given
    assert CALLS[op](n=0, pool=None, np=0) == B.OK
    if op == "attend":
        assert attend(heads=4 * 129) == B.ERR_UNSUPPORTED
        assert attend(new=[2 ** 31 - 1, 5, 0]) == B.ERR_UNSUPPORTED
        assert attend(new=[0, 0, 0], q=None, out=None) == B.OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="this check is for a box without a GPU")
def test_valid_calls_fail_loudly_without_a_device():
    for op in CALLS:
        assert CALLS[op]() == B.ERR_CUDA, op
    assert attend(out=P0) == B.ERR_CUDA                # in place
    assert attend(new=[5, 30, 0]) == B.ERR_CUDA        # more queries than tokens
    assert attend(qs=0) == B.ERR_CUDA                  # one query for all
    assert append(ks=0, vs=0) == B.ERR_CUDA
    assert copy(dst=1 << 40, to=[1, 2]) == B.ERR_CUDA  # another pool
    assert copy(tokens=[0, 32]) == B.ERR_CUDA
    assert L.ebrl_pages_check() == B.ERR_CUDA


def test_binding_refusals():
    pool, table = pg.new_pool(LAY, 2, device="cpu"), torch.zeros((1, 2), dtype=torch.int32)
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16)
    for bad in (pool, pool[:, :-1], pool.float()):     # host memory; not pages; not bytes
        with pytest.raises(ValueError):
            pg.attend(LAY, bad, table, q, [1], [1])
    with pytest.raises(B.EbrlError):
        pg.append(LAY._replace(head_dim=40), pool, table, q, q, [1], [1])
    with pytest.raises(TypeError):
        pg.new_pool(LAY._replace(dtype=torch.float16), 1, device="cpu")
    for bad in (table.long(), table[0], torch.zeros((2, 2), dtype=torch.int32)):
        with pytest.raises(ValueError):
            pg._table(bad, 1)
    with pytest.raises(ValueError):
        pg._fits(LAY, table, torch.tensor([65], dtype=torch.int32))
    with pytest.raises(ValueError):
        pg._counts([1], [1, 2])
    with pytest.raises(TypeError):
        pg._packed(LAY, q.float(), 4, "k")
    for bad in (q[0], q[:, :, :32], q.expand(3, 4, 64).transpose(0, 1)):
        with pytest.raises(ValueError):
            pg._packed(LAY, bad, 4, "k")


# ---- the book ----------------------------------------------------------------------------------------------------------

class Model:
    """The rules of the book, plainly: lists of pages, sharing found by looking through all of them."""

    def __init__(self, n_pages, T, n_seqs):
        self.n, self.T, self.len, self.rows = n_pages, T, [0] * n_seqs, [[] for _ in range(n_seqs)]

    def names(self, p):
        return sum(p in r for r in self.rows)

    def take(self):
        return next(p for p in range(self.n) if self.names(p) == 0)

    def used(self):
        return len({p for r in self.rows for p in r})

    def extend(self, seqs, lens):
        moves = []
        for s, v in zip(seqs, lens):
            if v > self.len[s] and self.len[s] % self.T and self.names(self.rows[s][-1]) > 1:
                p = self.take()
                moves.append((self.rows[s][-1], p, self.len[s] % self.T))
                self.rows[s][-1] = p
            while len(self.rows[s]) * self.T < v:
                self.rows[s].append(-2)
                self.rows[s][-1] = self.take()
            self.len[s] = v
        return moves

    def compact(self, room):
        moves, used = [], self.used()
        for high in range(self.n - 1, used - 1, -1):
            if len(moves) == room:
                break
            if self.names(high):
                low = self.take()
                fill = max(min(self.T, self.len[s] - j * self.T) for s, r in enumerate(self.rows) for j, p in enumerate(r) if p == high)
                moves.append((high, low, fill))
                self.rows = [[low if p == high else p for p in r] for r in self.rows]
        return moves


def as_list(moves):
    return list(zip(*[m.tolist() for m in moves]))


@pytest.mark.parametrize("seed", range(8))
def test_book_is_the_model(seed):
    rng = random.Random(seed)
    T, n_pages, n_seqs = rng.choice([32, 64]), rng.choice([5, 70, 130]), 9
    book, model = pg.Book(n_pages, T, n_seqs), Model(n_pages, T, n_seqs)
    for step in range(120):
        what = rng.choice(["extend", "extend", "extend", "fork", "shorten", "compact", "clone"])
        if what == "extend":
            seqs = rng.sample(range(n_seqs), rng.randint(0, 3))
            lens = [model.len[s] + rng.choice([0, 1, rng.randint(0, T), rng.randint(0, 4 * T)]) for s in seqs]
            before = ([list(r) for r in model.rows], list(model.len))
            try:
                want = model.extend(seqs, lens)
            except StopIteration:      # not enough pages: nothing may have changed
                model.rows, model.len = before
                with pytest.raises(B.EbrlError) as e:
                    book.extend(seqs, lens)
                assert e.value.status == B.ERR_NOMEM
            else:
                assert as_list(book.extend(seqs, lens)) == want
        elif what == "fork":
            to = [s for s in range(n_seqs) if model.len[s] == 0][:rng.randint(0, 2)]
            frm = [rng.choice([s for s in range(n_seqs) if s not in to]) for _ in to]
            book.fork(frm, to)
            for a, b in zip(frm, to):
                model.rows[b], model.len[b] = list(model.rows[a]), model.len[a]
        elif what == "shorten":
            seqs = rng.sample(range(n_seqs), rng.randint(0, 2))
            lens = [rng.choice([0, rng.randint(0, model.len[s])]) for s in seqs]
            book.shorten(seqs, lens)
            for s, v in zip(seqs, lens):
                model.len[s], model.rows[s] = v, model.rows[s][:-(-v // T)]
        elif what == "compact":
            room = rng.choice([0, 1, 1000])
            assert as_list(book.compact(room)) == model.compact(room)
        else:
            other = book.clone()
            other.shorten(list(range(n_seqs)), 0)      # does not touch the first one
            assert other.used == 0
        assert book.used == model.used() and [book.len(s) for s in range(n_seqs)] == model.len
        width = max(1, max(len(r) for r in model.rows)) + 1
        assert book.table(list(range(n_seqs)), width).tolist() == [r + [-1] * (width - len(r)) for r in model.rows]
    book.compact()
    rows = [p for r in book.table(list(range(n_seqs))).tolist() for p in r if p >= 0]
    assert sorted(set(rows)) == list(range(book.used))


def test_book_refusals():
    book = pg.Book(4, 32, 3)
    book.extend([0], [40])
    assert len(book.extend([0], [40])[0]) == 0
    for fn in (lambda: book.extend([0], [39]), lambda: book.extend([3], [1]), lambda: book.extend([-1], [1]), lambda: book.extend([1, 1], [1, 2]),
               lambda: book.fork([0], [0]), lambda: book.fork([1], [0]), lambda: book.fork([0, 0], [1, 1]), lambda: book.fork([0, 1], [1, 2]), lambda: book.fork([0], [5]),
               lambda: book.shorten([0], 41), lambda: book.shorten([0], -1), lambda: book.shorten([0, 0], 0), lambda: book.compact(-1), lambda: book.table([0], 1),
               lambda: book.table([9])):
        with pytest.raises(B.EbrlError) as e:
            fn()
        assert e.value.status == B.ERR_INVALID_ARG and book.used == 2 and book.len(0) == 40 and book.len(1) == 0
    with pytest.raises(B.EbrlError) as e:
        book.extend([1, 2], [32, 64])
    assert e.value.status == B.ERR_NOMEM and book.used == 2
    with pytest.raises(ValueError):
        book.extend([0, 1], [50])
    assert book.len(7) == -1 and book.len(-1) == -1
    for args in ((-1, 32, 1), (1, 0, 1), (1, 32, -1)):
        with pytest.raises(B.EbrlError):
            pg.Book(*args)
    assert L.ebrl_pages_book_extend(None, 0, None, None, None, None, None, None) == B.ERR_INVALID_ARG
    assert L.ebrl_pages_book_clone(None, C.byref(C.c_void_p())) == B.ERR_INVALID_ARG
    assert L.ebrl_pages_book_len(None, 0) == -1
    assert pg.Book(0, 32, 0).table([]).shape == (0, 0)


def test_two_writers_of_one_shared_page_get_a_copy_but_the_last():
    """The parent and its two children extend in one call: two copies, the third keeps the page."""
    book = pg.Book(5, 32, 3)
    book.extend([0], [40])
    book.fork([0, 0], [1, 2])
    moves = book.extend([0, 1, 2], [41, 41, 41])
    assert as_list(moves) == [(1, 2, 8), (1, 3, 8)]
    assert book.table([0, 1, 2]).tolist() == [[0, 2], [0, 3], [0, 1]] and book.used == 4
