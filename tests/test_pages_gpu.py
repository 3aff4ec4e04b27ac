"""GPU tests of the operators on paged caches against plain implementations in 64 bits.

Tolerances of attend, derived from the arithmetic.  A score is an fp32 sum of hd products; the tensor core may truncate, so it is off by at
most E = 4 hd 2^-23 max_t(|scale| sum |q| |k|) (bf16 products are exact; of fp32 operands in two tf32 terms, the first rounded to 11 bits, the second
cut to 11 bits, 2^-11 * 2^-10 of each operand is lost and 2^-11 * 2^-11 for the product of the second terms: 5 * 2^-22 more).  A weight is then off by a factor 1 + E + 2^-21 (ex2 and the fold of the two
factors into its argument; exp of a difference of E).  Sums over N tokens are joined from N / 8 steps of up to three products: S = (3 N / 8 + 64) 2^-23
of the sum of the absolute values.  bf16 weights are rounded (2^-8); fp32 ones lose 5 * 2^-22 as above.  With A = sum_t w_t |v_t| (w the
softmax weights) the result is off by A (2 (E + 2^-21) + 2 S + 2^-8 or 5 * 2^-22) and its own rounding, 2^-8 or 2^-24 of it.
lse: E + S + 2^-21 (1 + |lse|)."""
import math

import pytest
import torch

from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import pages as pg
from paper_2609_27547_b200 import prefix8 as p8

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32


class Cache:
    """A pool of pages in random order, every element NaN but those of visible tokens within the lengths; what they are is known."""

    def __init__(self, lay, lens, hide=0.0, seed=0, lost=0.0, spare=2, poison=True, spread=0.4):
        g = torch.Generator().manual_seed(seed)
        T, n = lay.page_tokens, len(lens)
        counts = [-(-v // T) for v in lens]
        self.lay, self.lens, self.n_pages = lay, list(lens), sum(counts) + spare
        order = torch.randperm(self.n_pages, generator=g).tolist()
        width = max(counts + [1]) + 1
        self.rows = [[order.pop() for _ in range(c)] for c in counts]
        table = torch.full((n, width), -1, dtype=torch.int32)
        pool = pg.new_pool(lay, self.n_pages, device="cpu")
        elems, words = pg.views(lay, pool)
        if poison:
            elems.fill_(math.nan)
            words.fill_(-1)
        self.kv, self.see = [], []           # [kv_layers, 2, heads, len, hd] in 64 bits; truth values
        for i, v in enumerate(lens):
            x = torch.randn((lay.kv_layers, 2, lay.n_kv_heads, v, lay.head_dim), generator=g) * torch.exp(spread * torch.randn((lay.kv_layers, 2, lay.n_kv_heads, 1, lay.head_dim), generator=g))
            x = x.to(lay.dtype)
            see = torch.rand(v, generator=g) >= hide
            if hide and n > 2 and i == n // 2:
                see[:] = False
            for j, p in enumerate(self.rows[i]):
                table[i, j] = p
                if torch.rand((), generator=g) < lost:       # the page is not there: any number that is none of a page's
                    table[i, j] = [-1, self.n_pages, 2 ** 31 - 1, -2 ** 31][int(torch.randint(4, (), generator=g))]
                    see[j * T:(j + 1) * T] = False
                    continue
                k = min(T, v - j * T)
                part = see[j * T:j * T + k]
                at = torch.nonzero(part).flatten()
                elems[p][:, :, :, at] = x[:, :, :, j * T + at]
                bits = torch.ones(T, dtype=torch.bool)
                bits[:k] = part
                w = (bits.view(-1, 32).long() << torch.arange(32)).sum(-1)
                words[p] = torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)
            self.kv.append(x.double())
            self.see.append(see)
        self.pool, self.table = pool.cuda(), table.cuda()


def reference(cache, i, layer, q, scale, causal=True, window=0):
    """(out, lse, weighted absolute values, bound of a score's size) for the queries q [m, heads, hd] of sequence i, in 64 bits."""
    lay, n, m = cache.lay, cache.lens[i], q.shape[0]
    G = q.shape[1] // lay.n_kv_heads
    kv, see = cache.kv[i][layer].cuda(), cache.see[i].cuda()
    k, v = (x[:, see].repeat_interleave(G, 0) for x in kv)                   # [heads, visible, hd]
    pos = torch.nonzero(see).flatten()
    me = torch.arange(n - m, n, device="cuda")[:, None]
    ok = torch.ones((m, len(pos)), dtype=torch.bool, device="cuda")
    if causal:
        ok &= pos <= me
        if window:
            ok &= pos > me - window
    x = q.double().transpose(0, 1)                                             # [heads, m, hd]
    s = scale * (x @ k.transpose(1, 2))
    size = float((abs(scale) * (x.abs() @ k.abs().transpose(1, 2))).max()) if s.numel() else 0.0
    s = s.masked_fill(~ok, -math.inf)
    lse = torch.logsumexp(s, -1)
    w = torch.where(lse[..., None] > -math.inf, torch.exp(s - lse[..., None]), 0.0)
    return (w @ v).transpose(0, 1), lse.transpose(0, 1), (w @ v.abs()).transpose(0, 1), size


def check(cache, layer, q, new, out, lse, scale=None, causal=True, window=0):
    lay = cache.lay
    scale = 1 / math.sqrt(lay.head_dim) if scale is None else scale
    f32, at, worst = lay.dtype is F, 0, 0.0
    for i, m in enumerate(new):
        if m == 0:
            continue
        o, l, a, size = reference(cache, i, layer, q[at:at + m], scale, causal, window)
        E = 4 * lay.head_dim * 2.0 ** -23 * size + (5 * 2.0 ** -22 * size if f32 else 0)
        S = (3 * cache.lens[i] / 8 + 64) * 2.0 ** -23
        tol = a * (2 * (E + 2.0 ** -21) + 2 * S + (5 * 2.0 ** -22 if f32 else 2.0 ** -8)) + o.abs() * (2.0 ** -24 if f32 else 2.0 ** -8) + 1e-37
        got, got_l = out[at:at + m].double(), lse[at:at + m].double()
        empty = l == -math.inf
        assert (got[empty] == 0).all() and (got_l[empty] == -math.inf).all(), i
        off = (got - o).abs() / tol
        assert not off.isnan().any() and float(off.max()) <= 1, (i, float(off.max()))
        worst = max(worst, float(off.max()))
        full = ~empty
        assert ((got_l - l).abs()[full] <= E + S + 2.0 ** -21 * (1 + l[full].abs())).all(), i
        at += m
    return worst


def queries(lay, rows, G, seed=0, size=1.3):
    g = torch.Generator().manual_seed(seed + 77)
    return (size * torch.randn((rows, lay.n_kv_heads * G, lay.head_dim), generator=g)).to(lay.dtype).cuda()


LENS = [0, 1, 31, 32, 33, 64, 65, 100, 130, 300, 17, 5]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T", [32, 64, 256])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, F])
def test_attend_ragged_hidden_lost_pages(dtype, hd, T, causal):
    lay = pg.Layout(2, 2, hd, T, dtype)
    cache = Cache(lay, LENS, hide=0.3, lost=0.1, seed=hd + T)
    for G, counts in ((1, [1] * len(LENS)), (3, [3, 1, 0, 32, 33, 5, 7, 100, 2, 129, 20, 5])):
        q = queries(lay, sum(counts), G, seed=T)
        for split in (0, -1, 128):
            out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, LENS, layer=1, causal=causal, split_tokens=split)
            check(cache, 1, q, counts, out, lse, causal=causal)


@pytest.mark.parametrize("window", [1, 2, 31, 33, 100, 10 ** 6])
@pytest.mark.parametrize("dtype,hd", [(BF, 128), (BF, 64), (F, 32), (F, 128)])
def test_attend_window(dtype, hd, window):
    lay = pg.Layout(1, 2, hd, 32, dtype)
    lens, counts = [700, 40, 3, 1000, 129], [1, 40, 5, 300, 128]
    cache = Cache(lay, lens, hide=0.1, seed=window % 97)
    q = queries(lay, sum(counts), 2, seed=hd)
    for split in (0, 128):
        out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, lens, window=window, split_tokens=split)
        check(cache, 0, q, counts, out, lse, window=window)


@pytest.mark.parametrize("dtype,hd,m", [(BF, 64, 1), (BF, 128, 20), (BF, 128, 90), (BF, 32, 300), (F, 64, 40)])
def test_attend_tokens_before_every_window_may_hold_anything(dtype, hd, m):
    lay = pg.Layout(1, 2, hd, 64, dtype)
    lens, window = [900, 450], 37
    cache = Cache(lay, lens, seed=m)
    elems, _ = pg.views(lay, cache.pool)
    for i, n in enumerate(lens):
        for t in range(n - m - window + 1):
            elems[cache.rows[i][t // 64], :, :, :, t % 64] = math.nan if t % 2 else math.inf
    q = queries(lay, 2 * m, 2, seed=1)
    for split in (0, 128):
        out, lse = pg.attend(lay, cache.pool, cache.table, q, [m, m], lens, window=window, split_tokens=split)
        check(cache, 0, q, [m, m], out, lse, window=window)


@pytest.mark.parametrize("G,m", [(1, 1), (1, 16), (1, 17), (2, 8), (7, 3), (8, 4), (5, 13), (128, 1), (64, 5), (1, 64), (4, 33), (3, 128), (1, 257)])
@pytest.mark.parametrize("dtype", [BF, F])
def test_attend_rows_of_shared_heads(dtype, G, m):
    lay = pg.Layout(1, 2, 64, 64, dtype)
    lens = [400, 277, m]
    cache = Cache(lay, lens, seed=G)
    q = queries(lay, 3 * m, G, seed=m)
    out, lse = pg.attend(lay, cache.pool, cache.table, q, [m] * 3, lens)
    check(cache, 0, q, [m] * 3, out, lse)


@pytest.mark.parametrize("dtype,hd", [(BF, 128), (BF, 64), (BF, 32), (F, 64)])
def test_attend_long_sequences_are_cut(dtype, hd):
    lay = pg.Layout(1, 2, hd, 128, dtype)
    lens, counts = [20001, 9000, 50, 0], [1, 8, 3, 2]
    cache = Cache(lay, lens, hide=0.2, seed=3)
    q = queries(lay, sum(counts), 4, seed=5)
    for split in (0, -1, 512, 9088):
        out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, lens, split_tokens=split)
        check(cache, 0, q, counts, out, lse)


@pytest.mark.parametrize("dtype", [BF, F])
def test_attend_under_a_quota(dtype):
    lay = pg.Layout(1, 4, 64, 32, dtype)
    lens = [(37 * i) % 500 for i in range(40)] + [5000]
    counts = [1 + i % 40 for i in range(41)]
    cache = Cache(lay, lens, seed=9)
    q = queries(lay, sum(counts), 2)
    for quota in (1, 16, 74):
        out, lse = pg.attend(lay, cache.pool, cache.table, q, counts, lens, sm_quota=quota)
        check(cache, 0, q, counts, out, lse)
    with pytest.raises(B.EbrlError) as e:
        pg.attend(lay, cache.pool, cache.table, q, counts, lens, sm_quota=10 ** 6)
    assert e.value.status == B.ERR_QUOTA


@pytest.mark.parametrize("m", [1, 40])
@pytest.mark.parametrize("dtype,hd", [(BF, 64), (BF, 128), (F, 64)])
def test_attend_alone_or_in_company_is_the_same_bit_for_bit_when_nothing_is_divided(dtype, hd, m):
    lay = pg.Layout(1, 2, hd, 32, dtype)
    lens = [(211 * i) % 700 + 1 for i in range(1100)]            # more than one launch takes
    cache = Cache(lay, lens, seed=4)
    q = queries(lay, m * len(lens), 2)
    out, lse = pg.attend(lay, cache.pool, cache.table, q, [m] * len(lens), lens, split_tokens=-1)
    for i in (0, 1, 500, 1023, 1024, 1099):
        one, one_l = pg.attend(lay, cache.pool, cache.table[i:i + 1], q[i * m:(i + 1) * m], [m], lens[i:i + 1], split_tokens=-1)
        assert torch.equal(one, out[i * m:(i + 1) * m]) and torch.equal(one_l, lse[i * m:(i + 1) * m])
        lone = Cache.__new__(Cache)
        lone.lay, lone.lens, lone.kv, lone.see = lay, lens[i:i + 1], cache.kv[i:i + 1], cache.see[i:i + 1]
        check(lone, 0, q[i * m:(i + 1) * m], [m], one, one_l)


@pytest.mark.parametrize("m", [3, 80])
@pytest.mark.parametrize("dtype", [BF, F])
def test_attend_strides_in_place_and_rows_behind_the_last_query(dtype, m):
    lay = pg.Layout(1, 2, 64, 32, dtype)
    lens, counts = [300, 90], [m, m + 2]
    total, heads = sum(counts), 4
    cache = Cache(lay, lens, seed=8)
    wide = torch.randn((total + 3, 3 * heads, 64), generator=torch.Generator().manual_seed(1)).to(dtype).cuda()    # queries, keys, values of one projection
    q = wide[:, :heads]
    want, want_l = pg.attend(lay, cache.pool, cache.table, q[:total].contiguous(), counts, lens)
    check(cache, 0, q[:total], counts, want, want_l)
    out, lse = torch.full((total + 3, 2 * heads, 64), 7.0, dtype=dtype, device="cuda"), torch.full((total + 3, heads), 7.0, device="cuda")
    pg.attend(lay, cache.pool, cache.table, q, counts, lens, out=out[:, heads:], lse=lse)
    assert torch.equal(out[:total, heads:], want) and torch.equal(lse[:total], want_l)
    assert (out[:, :heads] == 7).all() and (out[total:] == 7).all() and (lse[total:] == 7).all()
    before = wide.clone()
    pg.attend(lay, cache.pool, cache.table, q, counts, lens, out=q)
    assert torch.equal(wide[:total, :heads], want) and torch.equal(wide[:, heads:], before[:, heads:]) and torch.equal(wide[total:], before[total:])
    # one query for all rows
    same = before[:1, :heads].expand(total, heads, 64)
    out, lse = pg.attend(lay, cache.pool, cache.table, same, counts, lens)
    check(cache, 0, same, counts, out, lse)


def test_attend_scales_and_large_scores():
    lay = pg.Layout(1, 1, 64, 32, BF)
    cache = Cache(lay, [200, 64], seed=2)
    for m in (4, 64):
        q = queries(lay, 2 * m, 2, size=20.0)
        for scale in (0.0, -0.2, 0.125, 3.0):
            out, lse = pg.attend(lay, cache.pool, cache.table, q, [m, m], cache.lens, scale=scale)
            check(cache, 0, q, [m, m], out, lse, scale=scale)


# ---- append ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("dtype,hd,T", [(BF, 32, 32), (BF, 128, 256), (F, 64, 64), (F, 128, 32)])
def test_append_writes_its_tokens_and_nothing_else(dtype, hd, T, masked):
    lay = pg.Layout(2, 3, hd, T, dtype)
    lens = [(29 * i) % 400 + 1 for i in range(60)] + [0, 1, 2 * T]
    new = [min(v, (53 * i) % 130) for i, v in enumerate(lens)]
    cache = Cache(lay, lens, hide=0.3, seed=1)
    table = cache.table.clone()
    table[3, 0] = -1
    table[9, 1] = cache.n_pages
    total = sum(new)
    g = torch.Generator().manual_seed(5)
    wide = torch.randn((total + 1, 11, hd), generator=g).to(dtype).cuda()
    k, v = wide[:, 1:4], wide[:, 6:9]
    mask = (torch.rand(total + 1, generator=g) > 0.4) if masked else None
    want = cache.pool.cpu().clone()
    elems, words = pg.views(lay, want)
    bits = ((words[:, torch.arange(T) // 32] >> (torch.arange(T) % 32)) & 1).bool()
    rows, at = table.cpu().tolist(), 0
    for i, (n, m) in enumerate(zip(lens, new)):
        for j in range(m):
            t = n - m + j
            p = rows[i][t // T]
            if 0 <= p < cache.n_pages:
                see = mask is None or bool(mask[at])
                elems[p, 1, 0, :, t % T] = k[at].cpu() if see else 0
                elems[p, 1, 1, :, t % T] = v[at].cpu() if see else 0
                bits[p, t % T] = see
            at += 1
    w = (bits.view(len(bits), -1, 32).long() << torch.arange(32)).sum(-1)
    words.copy_(torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32))
    start = cache.pool.clone()
    for quota in (0, 5):
        cache.pool.copy_(start)
        pg.append(lay, cache.pool, table, k, v, new, lens, layer=1, mask=None if mask is None else (mask.cuda() if quota else mask.to(torch.uint8).cuda()), sm_quota=quota)
        assert torch.equal(cache.pool.cpu(), want)


def test_append_more_sequences_than_one_launch_takes():
    lay = pg.Layout(1, 1, 32, 32, BF)
    n = 2500
    pool = pg.new_pool(lay, n)
    table = torch.arange(n, dtype=torch.int32).flip(0).reshape(n, 1).cuda()
    x = torch.randn((n, 1, 32), generator=torch.Generator().manual_seed(0)).to(BF).cuda()
    pg.append(lay, pool, table, x, -x, [1] * n, [1 + i % 32 for i in range(n)])
    elems, words = pg.views(lay, pool)
    slot = (torch.arange(n) % 32).cuda()
    page = table[:, 0].long()
    assert torch.equal(elems[page, 0, 0, 0, slot], x[:, 0]) and torch.equal(elems[page, 0, 1, 0, slot], -x[:, 0])
    assert torch.equal(words[page, 0].long() & 0xffffffff, 1 << slot.long()) and int((elems != 0).any(-1).sum()) == 2 * n


# ---- copy --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,hd,T,layers", [(BF, 32, 32, 1), (BF, 128, 64, 2), (F, 64, 256, 1), (F, 128, 128, 3)])
def test_copy_is_exact_and_leaves_the_rest(dtype, hd, T, layers):
    lay = pg.Layout(layers, 3, hd, T, dtype)
    n = 12
    g = torch.Generator().manual_seed(3)
    src, other = (torch.randint(0, 256, (n, lay.page_bytes), dtype=torch.uint8, generator=g) for _ in range(2))
    frm, to, tokens = [0, 0, 3, 11, 4, 5], [1, 2, 10, 9, 8, 7], [T, 1, 31, T - 1, 0, 33 % T]
    e0, w0 = pg.views(lay, src)
    for within in (True, False):
        want = (src if within else other).clone()
        e1, w1 = pg.views(lay, want)
        for a, b, k in zip(frm, to, tokens):
            e1[b][:, :, :, :k] = e0[a][:, :, :, :k]
            for w in range(T // 32):
                m = (1 << min(32, max(0, k - 32 * w))) - 1
                v = (int(w1[b, w]) & ~m & 0xffffffff) | (int(w0[a, w]) & m)
                w1[b, w] = v - 2 ** 32 if v >= 2 ** 31 else v
        for quota in (0, 3):
            dev = src.cuda()
            dst = dev if within else other.cuda()
            pg.copy(lay, dev, dst, (frm, to, tokens), sm_quota=quota)
            ge, gw = pg.views(lay, dst.cpu())
            assert torch.equal(ge.contiguous().view(torch.uint8), e1.contiguous().view(torch.uint8)) and torch.equal(gw, w1)
            if not within:
                assert torch.equal(dev.cpu(), src)
    dev = src.cuda()
    pg.copy(lay, dev, dev, ([0], [5]))
    e, w = pg.views(lay, dev.cpu())
    assert torch.equal(e[5].contiguous().view(torch.uint8), e0[0].contiguous().view(torch.uint8)) and torch.equal(w[5], w0[0])


def test_copy_more_pages_than_one_launch_takes():
    lay = pg.Layout(1, 1, 32, 32, BF)
    n = 5000
    src = torch.randint(0, 256, (n, lay.page_bytes), dtype=torch.uint8, generator=torch.Generator().manual_seed(0)).cuda()
    dst = torch.zeros_like(src)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    pg.copy(lay, src, dst, (torch.arange(n, dtype=torch.int32), order))
    nb = 2 * 32 * 32 * 2 + 4
    assert torch.equal(dst[order.long().cuda(), :nb], src[:, :nb])


# ---- gather ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,hd,T", [(BF, 32, 32), (BF, 128, 256), (F, 64, 64), (F, 128, 32)])
def test_gather_is_the_planes_of_the_visible_tokens(dtype, hd, T):
    lay = pg.Layout(2, 3, hd, T, dtype)
    lens = [0, 1, 31, 32, 33, 300, 64, 200]
    cache = Cache(lay, lens, hide=0.3, lost=0.2, seed=6)
    n, d = len(lens), 3 * hd

    def want(i):
        x = cache.kv[i] * cache.see[i][:, None]
        return torch.where(cache.see[i][:, None], x, torch.zeros(())).permute(0, 1, 3, 2, 4).flatten(3).to(dtype)

    for quota in (0, 4):
        planes = pg.gather(lay, cache.pool, cache.table, lens, sm_quota=quota)
        for i in range(n):
            assert torch.equal(planes[i].cpu(), want(i))
        wide = torch.full((n, 2, 2, 310, d + 64), 7.0, dtype=dtype, device="cuda")
        seen = torch.full((n, 305), 9, dtype=torch.uint8, device="cuda")
        pg.gather(lay, cache.pool, cache.table, lens, wide[:, :, :, :, 32:32 + d], mask=seen, sm_quota=quota)
        for i, v in enumerate(lens):
            assert torch.equal(wide[i, :, :, :v, 32:32 + d].cpu(), want(i)) and (wide[i, :, :, v:] == 7).all()
            assert torch.equal(seen[i, :v].cpu().bool(), cache.see[i]) and (seen[i, v:] == 9).all()
        assert (wide[..., :32] == 7).all() and (wide[..., 32 + d:] == 7).all()
    masks = [torch.full((v,), 9, dtype=torch.uint8, device="cuda") if i % 2 else None for i, v in enumerate(lens)]
    pg.gather(lay, cache.pool, cache.table, lens, planes, mask=masks)
    assert all(m is None or torch.equal(m.cpu().bool(), cache.see[i]) for i, m in enumerate(masks))


def test_gather_more_sequences_than_one_launch_takes():
    lay = pg.Layout(1, 1, 32, 32, F)
    lens = [1 + i % 40 for i in range(1500)]
    cache = Cache(lay, lens, seed=1)
    planes = torch.zeros((1500, 1, 2, 40, 32), device="cuda")
    pg.gather(lay, cache.pool, cache.table, lens, planes)
    for i in (0, 700, 1023, 1024, 1499):
        assert torch.equal(planes[i, 0, :, :lens[i]].cpu(), cache.kv[i][0, :, 0].float()) and (planes[i, 0, :, lens[i]:] == 0).all()


# ---- together, and as a program uses them --------------------------------------------------------------------------------

def dense(q, k, v, scale, causal):
    """One sequence in 64 bits: q [m, heads, hd] against k, v [heads, n, hd], the queries being the last m tokens."""
    m, n = q.shape[0], k.shape[1]
    G = q.shape[1] // k.shape[0]
    s = scale * (q.double().transpose(0, 1) @ k.double().repeat_interleave(G, 0).transpose(1, 2))
    if causal:
        s = s.masked_fill(torch.arange(n, device=s.device) > torch.arange(n - m, n, device=s.device)[:, None], -math.inf)
    return (torch.softmax(s, -1) @ v.double().repeat_interleave(G, 0)).transpose(0, 1)


@pytest.mark.parametrize("dtype", [BF, F])
def test_histories_grow_fork_are_compacted_and_reach_the_action_head(dtype):
    """Two episodes start, grow, branch into children that go on by themselves, one is reset, the pool is compacted; every chunk's attention is what the
    dense history gives.  The histories, gathered, are planes that a handle takes: its chunks are those of the dense planes bit for bit."""
    from paper_2609_27547_b200 import synth
    w = synth.scaled(synth.WORKLOADS[0], B=4, dtype="bf16" if dtype is BF else "f32", d=256, P=(16, 200))
    heads, hd, T, layers = w.n_heads, w.d // w.n_heads, 32, 2
    lay = pg.Layout(layers, heads, hd, T, dtype)
    book, pool = pg.Book(60, T, 6), pg.new_pool(lay, 60)
    pool[:, :] = 0x7f                          # whatever a pool holds at first
    g = torch.Generator().manual_seed(1)
    hist = {s: torch.zeros((layers, 2, heads, 0, hd), dtype=dtype, device="cuda") for s in range(6)}

    def step(seqs, new):
        lens = [book.len(s) + k for s, k in zip(seqs, new)]
        pg.copy(lay, pool, pool, book.extend(seqs, lens))
        table = book.table(seqs, device="cuda")
        total = sum(new)
        for l in range(layers):
            qkv = torch.randn((total, 3 * heads, hd), generator=g).to(dtype).cuda()
            q, k, v = qkv[:, :heads], qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
            pg.append(lay, pool, table, k, v, new, lens, layer=l)
            at = 0
            for s, n in zip(seqs, new):
                if l == 0:
                    hist[s] = torch.cat([hist[s], torch.zeros((layers, 2, heads, n, hd), dtype=dtype, device="cuda")], 3)
                hist[s][l, 0, :, hist[s].shape[3] - n:] = k[at:at + n].transpose(0, 1)
                hist[s][l, 1, :, hist[s].shape[3] - n:] = v[at:at + n].transpose(0, 1)
                at += n
            out, _ = pg.attend(lay, pool, table, q, new, lens, layer=l)
            at = 0
            for s, n in zip(seqs, new):
                want = dense(q[at:at + n], hist[s][l, 0], hist[s][l, 1], 1 / math.sqrt(hd), True)
                off = (out[at:at + n].double() - want).abs().max()
                # |values| <= 5 and scores' absolute sums <= 8: twice 5 * 2^-8 and twice 5 E, E = 4 * 64 * 2^-23 * 8
                assert float(off) <= (10 * 2.0 ** -8 if dtype is BF else 0.0) + 10 * 2.0 ** -12, (s, l, float(off))
                at += n

    step([0, 1], [50, 20])
    step([0, 1], [1, 13])
    book.fork([0, 0, 1], [2, 3, 4])
    for a, b in ((0, 2), (0, 3), (1, 4)):
        hist[b] = hist[a].clone()
    step([0, 2, 3, 4], [1, 40, 1, 2])           # the parent goes on, too
    book.shorten([0], 0)
    hist[0] = hist[0][:, :, :, :0]
    pg.copy(lay, pool, pool, book.compact())
    step([1, 2, 3, 4], [5, 1, 64, 1])
    step([0, 3], [3, 1])
    seqs = [1, 2, 3, 4]
    lens = [book.len(s) for s in seqs]
    planes = pg.gather(lay, pool, book.table(seqs, device="cuda"), lens)
    for s, x in zip(seqs, planes):
        assert torch.equal(x, hist[s].permute(0, 1, 3, 2, 4).flatten(3))
    pg.check()
    cfg = dict(max_group_envs=4)
    outs = []
    for kv in (planes, [hist[s].permute(0, 1, 3, 2, 4).flatten(3).contiguous() for s in seqs]):
        gen = B.ActGen(B.cfg_for(w, **cfg), synth.make_weights(w))
        noise = torch.stack([synth.make_env(w, e).noise for e in range(4)]).cuda()
        out = torch.empty_like(noise)
        gen.submit([0, 1, 2, 3], [x[:1].contiguous() for x in kv], noise, out)
        gen.sync()
        gen.destroy()
        outs.append(out)
    assert torch.equal(*outs) and bool(torch.isfinite(outs[0]).all())


def test_gathered_histories_with_hidden_tokens_become_records():
    lay = pg.Layout(1, 4, 64, 32, BF)
    lens = [100, 33, 64]
    cache = Cache(lay, lens, hide=0.3, seed=3)
    seen = torch.zeros((3, 100), dtype=torch.uint8, device="cuda")
    planes = pg.gather(lay, cache.pool, cache.table, lens, torch.zeros((3, 1, 2, 100, 256), dtype=BF, device="cuda"), mask=seen)
    rec = p8.Layout(1, 4, 64, 100)
    a, b = p8.new_pool(rec, 3), p8.new_pool(rec, 3)
    p8.quantize(rec, a, planes, lens, mask=seen)
    p8.quantize(rec, b, [x.permute(0, 1, 3, 2, 4).flatten(3).to(BF).cuda() for x in cache.kv], lens, mask=[s.to(torch.uint8).cuda() for s in cache.see])
    assert torch.equal(a, b)


def test_captured_and_replayed_on_other_pages_and_data():
    """One graph: append, attend of a mixed batch (several kernels side by side, and pieces), gather.  The replay reads tables, pools and inputs as they are then."""
    lay = pg.Layout(1, 4, 64, 32, BF)
    lens, new = [3000, 500, 40, 900], [1, 200, 40, 20]
    total = sum(new)
    states = []
    for seed in (1, 2):
        c = Cache(lay, lens, seed=seed)
        g = torch.Generator().manual_seed(seed)
        states.append((c, torch.randn((total, 12, 64), generator=g).to(BF).cuda()))
    pool, table, qkv = states[0][0].pool.clone(), states[0][0].table.clone(), states[0][1].clone()
    planes = [torch.zeros((1, 2, n, 256), dtype=BF, device="cuda") for n in lens]

    def run():
        pg.append(lay, pool, table, qkv[:, 4:8], qkv[:, 8:], new, lens)
        out, lse = pg.attend(lay, pool, table, qkv[:, :4], new, lens)
        pg.gather(lay, pool, table, lens, planes)
        return out, lse
    run()                                       # (kernel attributes are set at the first call)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = run()
    for c, x in states[::-1] + states:
        pool.copy_(c.pool)
        table.copy_(c.table)
        qkv.copy_(x)
        graph.replay()
        got = [t.clone() for t in (out, lse, *planes)]
        torch.cuda.synchronize()
        pool.copy_(c.pool)
        eager = run()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1]) and all(torch.equal(a, b) for a, b in zip(got[2:], planes))
    del graph


def test_two_streams_and_a_stream_that_is_not_current():
    lay = pg.Layout(1, 4, 128, 64, BF)
    lens, new = [2500, 700, 300], [1, 100, 30]
    cache = Cache(lay, lens, seed=5)
    q = queries(lay, sum(new), 2)
    want, want_l = pg.attend(lay, cache.pool, cache.table, q, new, lens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    results = []
    for _ in range(10):
        for s in streams:
            results.append(pg.attend(lay, cache.pool, cache.table, q, new, lens, stream=s))
    torch.cuda.synchronize()
    for out, lse in results:
        assert torch.equal(out, want) and torch.equal(lse, want_l)
    pg.check()


@pytest.mark.parametrize("dtype", [BF, F])
def test_pages_behind_four_gigabytes(dtype):
    lay = pg.Layout(1, 16, 128, 256, dtype)
    n_pages = int(4.6e9 / lay.page_bytes) + 2
    pool = torch.zeros((n_pages, lay.page_bytes), dtype=torch.uint8, device="cuda")
    small = Cache(lay, [300, 520], seed=2, spare=0)
    high = [n_pages - 1 - p for p in range(small.n_pages)]
    pool[high] = small.pool
    table = torch.where(small.table >= 0, n_pages - 1 - small.table, small.table)
    for new in ([1, 1], [200, 3]):
        q = queries(lay, sum(new), 1)
        out, lse = pg.attend(lay, pool, table, q, new, [300, 520])
        want = pg.attend(lay, small.pool, small.table, q, new, [300, 520])
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    x = torch.randn((20, 16, 128), generator=torch.Generator().manual_seed(0)).to(dtype).cuda()
    pg.append(lay, pool, table, x, -x, [0, 20], [300, 520])
    pg.append(lay, small.pool, small.table, x, -x, [0, 20], [300, 520])
    assert torch.equal(pool[high], small.pool)
    pg.copy(lay, pool, pool, ([high[0]], [0]))
    e, _ = pg.views(lay, pool[[high[0], 0]])
    assert torch.equal(e[0].contiguous().view(torch.uint8), e[1].contiguous().view(torch.uint8))
    for a, b in zip(pg.gather(lay, pool, table, [300, 520]), pg.gather(lay, small.pool, small.table, [300, 520])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("seed", range(12))
def test_attend_random_calls(seed):
    import random
    rng = random.Random(seed)
    dtype = rng.choice([BF, BF, F])
    lay = pg.Layout(rng.randint(1, 2), rng.choice([1, 2, 3]), rng.choice([32, 64, 128]), rng.choice([32, 64, 128, 256]), dtype)
    n, G = rng.randint(1, 9), rng.choice([1, 2, 3, 6, 16])
    lens = [rng.choice([rng.randint(0, 40), rng.randint(0, 700), rng.randint(0, 3000)]) for _ in range(n)]
    new = [rng.choice([0, 1, rng.randint(1, 20), rng.randint(1, 300)]) for _ in range(n)]
    causal = rng.random() < 0.7
    window = rng.choice([0, 0, rng.randint(1, 400)]) if causal else 0
    cache = Cache(lay, lens, hide=rng.choice([0.0, 0.2]), lost=rng.choice([0.0, 0.1]), seed=seed)
    q = queries(lay, sum(new), G, seed=seed)
    layer = lay.kv_layers - 1
    for quota in (0, rng.randint(1, 100)):
        for split in (0, -1, 128 * rng.randint(1, 8)):
            out, lse = pg.attend(lay, cache.pool, cache.table, q, new, lens, layer=layer, causal=causal, window=window, split_tokens=split, sm_quota=quota)
            check(cache, layer, q, new, out, lse, causal=causal, window=window)


def test_scores_that_rise_along_a_sequence():
    """Each tile's scores lie far above those of the ones before it, so that references have to follow; and far below, so that later tiles count for nothing."""
    lay = pg.Layout(1, 1, 64, 64, BF)
    cache = Cache(lay, [1500], seed=6)
    elems, _ = pg.views(lay, cache.pool)
    ramp = torch.linspace(-60, 60, 1500)
    for rise in (1, -1):
        for t in range(1500):
            k = torch.zeros(64)
            k[0] = rise * ramp[t]
            k[1:] = cache.kv[0][0, 0, 0, t, 1:].float() * 0.1
            cache.kv[0][0, 0, 0, t] = k.to(BF).double()
        x = cache.kv[0][0, 0, 0].to(BF).cuda()
        for j, p in enumerate(cache.rows[0]):
            k = min(64, 1500 - 64 * j)
            elems[p, 0, 0, 0, :k] = x[64 * j:64 * j + k]
        for m in (1, 33, 300):
            q = queries(lay, m, 1)
            q[:, 0, 0] = 4.0
            for split in (0, 128):
                out, lse = pg.attend(lay, cache.pool, cache.table, q, [m], [1500], split_tokens=split, scale=1.0)
                check(cache, 0, q, [m], out, lse, scale=1.0)


def test_refusals_on_the_device():
    lay = pg.Layout(1, 2, 64, 32, BF)
    cache = Cache(lay, [40], seed=1)
    q = queries(lay, 3, 2)
    k = q[:, :2].contiguous()
    bad_values = (lambda: pg.attend(lay, cache.pool, cache.table, q, [4], [40]), lambda: pg.attend(lay, cache.pool, cache.table, q, [1], [129]),
                  lambda: pg.attend(lay, cache.pool, cache.table.cpu(), q, [1], [40]), lambda: pg.attend(lay, cache.pool, cache.table, q, [1], [40], lse=q),
                  lambda: pg.attend(lay, cache.pool, cache.table, q, [1], [40], out=q[:, :2]), lambda: pg.append(lay, cache.pool, cache.table, k, k[:1], [2], [40]),
                  lambda: pg.append(lay, cache.pool, cache.table, q, q, [2], [40]), lambda: pg.append(lay, cache.pool, cache.table, k, k, [2], [40], mask=torch.ones(1, device="cuda")),
                  lambda: pg.copy(lay, cache.pool, cache.pool, ([0], [1, 2])), lambda: pg.copy(lay, cache.pool, cache.pool.cpu(), ([0], [1])),
                  lambda: pg.gather(lay, cache.pool, cache.table, [40], torch.zeros((1, 1, 2, 39, 128), dtype=BF, device="cuda")),
                  lambda: pg.gather(lay, cache.pool, cache.table, [-1]), lambda: pg.gather(lay, cache.pool, cache.table, [40], [torch.zeros((1, 2, 40, 100), dtype=BF, device="cuda")]))
    for fn in bad_values:
        with pytest.raises(ValueError):
            fn()
    for fn in (lambda: pg.attend(lay, cache.pool, cache.table, q, [1], [40], window=3, causal=False), lambda: pg.attend(lay, cache.pool, cache.table, q, [1], [40], scale=math.inf),
               lambda: pg.attend(lay, cache.pool, cache.table, q, [1], [40], layer=1), lambda: pg.attend(lay, cache.pool, cache.table, q, [-1], [40]),
               lambda: pg.append(lay, cache.pool, cache.table, k, k, [3], [2]), lambda: pg.copy(lay, cache.pool, cache.pool, ([0], [0])),
               lambda: pg.copy(lay, cache.pool, cache.pool, ([0], [1], [33]))):
        with pytest.raises(B.EbrlError):
            fn()
    with pytest.raises(TypeError):
        pg.attend(lay, cache.pool, cache.table, q.float(), [1], [40])


@pytest.mark.parametrize("hd,m", [(128, 200), (128, 20), (64, 40), (32, 40)])
def test_a_wait_that_runs_out_is_noted_and_the_device_stays_usable(hd, m):
    lay = pg.Layout(1, 1, hd, 64, BF)
    cache = Cache(lay, [300], seed=1)
    q = queries(lay, m, 1)
    L = pg._load()
    pg.check()
    L.ebrl_pages_test_drop_copies(20_000_000)
    try:
        pg.attend(lay, cache.pool, cache.table, q, [m], [300])
    finally:
        L.ebrl_pages_test_drop_copies(0)
    with pytest.raises(B.EbrlError) as e:
        pg.check()
    assert e.value.status == B.ERR_TIMEOUT
    pg.check()                                  # it is told once
    out, lse = pg.attend(lay, cache.pool, cache.table, q, [m], [300])
    check(cache, 0, q, [m], out, lse)
    pg.check()
