"""GPU tests of the operators on 8-bit prefix records against tests/prefix8_reference.py (64 bits).

Tolerances, derived from the arithmetic: a row's scores are fp32 sums of hd exact f16 products, so they are off by at most
E = 4 hd 2^-23 max_t(scale sum |q| |k|) (the tensor core may truncate, and the fold of two factors rounds; fp32 queries in two f16
terms lose 2^-22 of each product more, which the factor 4 covers); a weight then is off by a factor 1 + E, the sum of N weights by
(N / 8 + 64) 2^-24.  Weights are rounded to f16 (2^-11) or held in two terms (2^-22) before they meet the values.  The result is rounded to bf16
(2^-8 of it) or fp32 (2^-24)."""
import math

import numpy as np
import pytest
import torch

import prefix8_reference as ref
from paper_2609_27547_b200 import prefix8 as p8

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def planes_of(lay, P, dtype, seed, spread=0.4):
    g = torch.Generator().manual_seed(seed)
    d = lay.n_kv_heads * lay.head_dim
    x = torch.randn((lay.kv_layers, 2, P, d), generator=g) * torch.exp(spread * torch.randn((lay.kv_layers, 2, 1, d), generator=g))
    return x.to(DT[dtype])


def decoded(lay, pool, slot, layer, length):
    """(keys, values [heads, length, hd] in 64 bits, visible [length]) of a record, from its bytes."""
    codes, scales, words = p8.views(lay, pool.cpu())
    rep = np.repeat(np.abs(scales[slot, layer].numpy()).astype(np.float64), 32, axis=-1)[..., :length, None]
    kv = ref.VALUES[codes[slot, layer, :, :, :length].numpy()] * rep
    bits = np.array([(int(words[slot, t // 32]) >> (t % 32)) & 1 for t in range(length)], dtype=bool)
    return kv[0], kv[1], bits


def rows_of(q, i, kh, G):
    """The query rows of key/value head kh: [H * G, hd] in 64 bits."""
    return q[i][:, kh * G:(kh + 1) * G].double().cpu().numpy().reshape(-1, q.shape[-1])


def check_attend(lay, pool, q, lens, out, lse, layer, scale, slots=None):
    n, H, heads, hd = q.shape
    G = heads // lay.n_kv_heads
    f32 = q.dtype == torch.float32
    for i in range(n):
        k, v, vis = decoded(lay, pool, slots[i] if slots else i, layer, lens[i])
        for kh in range(lay.n_kv_heads):
            o, ls, sa = ref.attend(rows_of(q, i, kh, G), k[kh][vis], v[kh][vis], scale)
            got = rows_of(out, i, kh, G)
            got_l = lse[i, :, kh * G:(kh + 1) * G].double().cpu().numpy().reshape(-1)
            if not vis.any():
                assert (got == 0).all() and np.isneginf(got_l).all()
                continue
            E = 4 * hd * 2.0 ** -23 * sa
            sums = (len(k[kh]) / 8 + 64) * 2.0 ** -24
            vmax = np.abs(v[kh][vis]).max()
            tol = np.abs(o) * (2.0 ** -24 if f32 else 2.0 ** -8) + (2 * E + 2 * sums + (2.0 ** -22 if f32 else 2.0 ** -11)) * vmax + 1e-30
            assert (np.abs(got - o) <= tol).all(), (i, kh, float((np.abs(got - o) / tol).max()))
            assert (np.abs(got_l - ls) <= E + sums + 2.0 ** -22 * (1 + np.abs(ls))).all(), (i, kh)


def filled(lay, lens, dtype="bf16", hide=0.0, seed=0, n_slots=None, slots=None, poison=True):
    """A pool whose records were written by quantize; every other byte is 0x7f (NaN as a code, as a scale, all visible)."""
    n = len(lens)
    pool = p8.new_pool(lay, n_slots or n)
    if poison:
        pool.fill_(0x7f)
        pool[:, -(-lay.record_bytes // 2):] = 0xff
    g = torch.Generator().manual_seed(seed + 999)
    planes = [planes_of(lay, max(P, 1), dtype, seed + 7 * i)[:, :, :P].cuda() for i, P in enumerate(lens)]
    masks = None
    if hide:
        masks = [(torch.rand(max(P, 1), generator=g) >= hide).to(torch.uint8).cuda() for P in lens]
        if n > 2:
            masks[n // 2].zero_()
    p8.quantize(lay, pool, planes, lens, mask=masks, slots=slots)
    return pool, planes, masks


# ---- quantize ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantize_is_the_definition_bit_for_bit(hd, dtype):
    lay = p8.Layout(2, 3, hd, 77)
    lens = [0, 1, 31, 32, 33, 64, 77, 5]
    n = len(lens)
    pool = p8.new_pool(lay, n)
    pool.fill_(0x55)
    before = pool.clone()
    planes, masks = [], []
    for i, P in enumerate(lens):
        x = planes_of(lay, max(P, 1), "f32", 11 * i, spread=3.0)[:, :, :P].clone()
        x = x.to(DT[dtype])
        if P > 3:
            x[0, 0, 1, 0], x[0, 1, 2, 1], x[1, 0, 3, 2] = math.inf, -math.inf, math.nan
            x[1, 1, :3] = 0.0
            x[0, 1, 0] *= 2.0 ** -120      # next to the smallest normal numbers
        if P > 40:
            x[1, 1, 32:] = 0.0             # a block of zeros
        m = (torch.rand(max(P, 1), generator=torch.Generator().manual_seed(i)) > 0.3).to(torch.uint8)
        if P > 8:
            x[:, :, 6][:] = math.nan       # hidden: whatever stands there
            m[6] = 0
        planes.append(x.cuda())
        masks.append(m.cuda() if i % 2 else None)
    p8.quantize(lay, pool, planes, lens, mask=masks)
    codes, scales, words = (t.cpu().numpy() for t in p8.views(lay, pool))
    codes0, scales0, words0 = (t.cpu().numpy() for t in p8.views(lay, before))
    for i, P in enumerate(lens):
        vis = masks[i].cpu().numpy()[:P] != 0 if masks[i] is not None else np.ones(P, bool)
        nb = -(-P // 32)
        for l in range(2):
            for p in range(2):
                for h in range(3):
                    x = planes[i][l, p, :, h * hd:(h + 1) * hd].double().cpu().numpy()
                    c, s = ref.quantize_head(x, vis)
                    got = codes[i, l, p, h]
                    nan = np.isnan(ref.VALUES[c])
                    assert (np.where(nan, got[:P] & 127, got[:P]) == np.where(nan, 127, c)).all(), (i, l, p, h)
                    assert (got[P:] == codes0[i, l, p, h, P:]).all()
                    assert (scales[i, l, p, h, :nb] == s.astype(np.float32)).all()
                    assert (scales[i, l, p, h, nb:].view(np.int32) == scales0[i, l, p, h, nb:].view(np.int32)).all()
        want = [sum(int(v) << b for b, v in enumerate(vis[32 * w:32 * w + 32])) for w in range(nb)]
        assert [int(w) & 0xffffffff for w in words[i, :nb]] == want
        assert (words[i, nb:] == words0[i, nb:]).all()


def test_quantize_strided_planes_slots_quota_and_many_environments():
    lay = p8.Layout(1, 2, 32, 40)
    n = 300                                 # more than one launch takes
    wide = torch.randn((n, 1, 2, 48, 128), generator=torch.Generator().manual_seed(1)).cuda()
    x = wide[:, :, :, :40, 32:96]           # rows 128 apart, planes 48 rows apart
    lens = [(7 * i) % 41 for i in range(n)]
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(2)).to(torch.int32)
    a, b = p8.new_pool(lay, n), p8.new_pool(lay, n)
    p8.quantize(lay, a, x, lens, slots=slots, sm_quota=5)
    p8.quantize(lay, b, [x[i, :, :, :lens[i]].contiguous() for i in range(n)], lens)
    assert torch.equal(a[slots.long().cuda()], b)
    p8.quantize(lay, a, x, lens, slots=slots, mask=torch.ones((n, 64), dtype=torch.bool, device="cuda")[:, :40])
    assert torch.equal(a[slots.long().cuda()], b)


# ---- attend -----------------------------------------------------------------------------------------------------------

SHAPES = [
    # H, G, kv heads, hd, lengths, capacity, kv_layers
    (1, 1, 2, 64, [1, 0, 32, 33, 100], 100, 1),
    (8, 1, 4, 64, [64, 257, 31], 300, 2),
    (7, 1, 3, 32, [5, 129, 128, 640], 650, 1),
    (16, 1, 2, 128, [768, 1, 95], 768, 1),
    (9, 1, 1, 64, [200, 64], 200, 1),
    (19, 1, 2, 32, [77, 300], 300, 2),
    (32, 1, 2, 128, [130, 33], 130, 1),
    (32, 2, 2, 64, [150, 3], 160, 1),       # 64 query rows: two row tiles
    (5, 8, 1, 128, [70, 290], 290, 1),      # 40 rows, the second tile partly filled
    (1, 4, 2, 128, [1500, 2], 1500, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,kvh,hd,lens,cap,layers", SHAPES)
def test_attend_against_64_bits(H, G, kvh, hd, lens, cap, layers, dtype):
    lay = p8.Layout(layers, kvh, hd, cap)
    for hide in (0.0, 0.5):
        pool, _, _ = filled(lay, lens, hide=hide, seed=H + hd)
        q = (1.5 * torch.randn((len(lens), H, kvh * G, hd), generator=torch.Generator().manual_seed(H))).to(DT[dtype]).cuda()
        out, lse = p8.attend(lay, pool, q, lens, layer=layers - 1)
        check_attend(lay, pool, q, lens, out, lse, layers - 1, 1 / math.sqrt(hd))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [1, 8, 16, 32])
def test_attend_rising_and_falling_scores(dtype, H):
    """Scores that climb by hundreds along the prefix (every tile moves the maximum), fall, or stay huge: the running maximum has to follow."""
    hd, P = 64, 1000
    lay = p8.Layout(1, 1, hd, P)
    ramp = torch.linspace(-1, 1, P)
    for seed, shape in enumerate([ramp, -ramp, torch.where(torch.arange(P) == 613, 1.0, -1.0), torch.ones(P)]):
        x = planes_of(lay, P, "f32", seed)
        x[0, 0] = 0.05 * x[0, 0]
        x[0, 0, :, 0] = 30 * shape
        pool = p8.new_pool(lay, 1)
        p8.quantize(lay, pool, [x.cuda()], [P])
        q = torch.randn((1, H, 1, hd), generator=torch.Generator().manual_seed(seed)).to(DT[dtype])
        q[..., 0] = torch.linspace(-40, 40, H)[None, :, None] if H > 1 else 40.0
        q = q.cuda()
        out, lse = p8.attend(lay, pool, q, [P])
        check_attend(lay, pool, q, [P], out, lse, 0, 1 / 8)


def test_attend_queries_of_any_size_and_scale():
    """A row's size does not matter: queries are brought to one power of two and back."""
    lay = p8.Layout(1, 2, 64, 200)
    pool, _, _ = filled(lay, [200] * 4, seed=3)
    base = torch.randn((4, 8, 2, 64), generator=torch.Generator().manual_seed(5))
    for dtype in ("bf16", "f32"):
        for e in (-100, -30, 0, 30, 100):
            q = (base * 2.0 ** e).to(DT[dtype]).cuda()
            out, lse = p8.attend(lay, pool, q, [200] * 4, scale=0.1 * 2.0 ** -e)
            check_attend(lay, pool, q, [200] * 4, out, lse, 0, 0.1 * 2.0 ** -e)
        q = base.to(DT[dtype]).cuda()
        for scale in (0.0, -0.2):
            out, lse = p8.attend(lay, pool, q, [200] * 4, scale=scale)
            check_attend(lay, pool, q, [200] * 4, out, lse, 0, scale)
        q[1, 2] = 0.0
        out, lse = p8.attend(lay, pool, q, [200] * 4)
        check_attend(lay, pool, q, [200] * 4, out, lse, 0, 1 / 8)


def test_attend_any_finite_scales():
    """Scales need not be powers of two, nor alike: neighbouring blocks 2^60 apart, zero."""
    lay = p8.Layout(1, 1, 64, 300)
    pool, _, _ = filled(lay, [300], seed=4, poison=False)
    _, scales, _ = p8.views(lay, pool)
    scales[0, 0, 0, 0, :] *= 1.37
    scales[0, 0, 1, 0, :] *= torch.tensor([3.0, 2.0 ** 60, 1e-20, 0.0, 1.5, 1.1, 2.0 ** -60, 1.0, 1.0, 1.0], device="cuda")
    for dtype in ("bf16", "f32"):
        q = torch.randn((1, 8, 1, 64), generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
        out, lse = p8.attend(lay, pool, q, [300])
        check_attend(lay, pool, q, [300], out, lse, 0, 1 / 8)


def test_attend_nan_reaches_only_who_sees_it():
    lay = p8.Layout(1, 2, 64, 96)
    lens = [96, 70]
    planes = [planes_of(lay, P, "f32", P) for P in lens]
    planes[0][0, 0, 10, 3] = math.nan                     # a key of environment 0, head 0
    q = torch.randn((2, 4, 2, 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    pool = p8.new_pool(lay, 2)
    p8.quantize(lay, pool, [x.cuda() for x in planes], lens)
    out, lse = p8.attend(lay, pool, q, lens)
    assert out[0, :, 0].isnan().all() and lse[0, :, 0].isnan().all()
    assert not out[0, :, 1].isnan().any() and not out[1].isnan().any()
    # hidden, the same token is harmless; so is a query that is not a number, to other rows
    m = torch.ones(96, dtype=torch.uint8)
    m[10] = 0
    p8.quantize(lay, pool, [x.cuda() for x in planes], lens, mask=[m.cuda(), None])
    out, lse = p8.attend(lay, pool, q, lens)
    check_attend(lay, pool, q, lens, out, lse, 0, 1 / 8)
    q2 = q.clone()
    q2[0, 1, 0, 5] = math.nan
    out2, _ = p8.attend(lay, pool, q2, lens)
    assert out2[0, 1, 0].isnan().all()
    keep = torch.ones((2, 4, 2), dtype=torch.bool)
    keep[0, 1, 0] = False
    assert torch.equal(out2[keep.cuda()], out[keep.cuda()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_does_not_depend_on_company_order_or_quota(dtype):
    lay = p8.Layout(1, 2, 128, 500)
    lens = [500, 1, 33, 260, 0, 128, 499, 64]
    pool, _, _ = filled(lay, lens, hide=0.2)
    q = torch.randn((8, 16, 2, 128), generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
    out, lse = p8.attend(lay, pool, q, lens, split_tokens=-1)
    for quota in (1, 3, 37, 148):
        o, l = p8.attend(lay, pool, q, lens, split_tokens=-1, sm_quota=quota)
        assert torch.equal(o, out) and torch.equal(l, lse)
    perm = [5, 0, 7, 3, 3, 1]                              # a slot may be read twice
    o, l = p8.attend(lay, pool, q[perm].contiguous(), [lens[i] for i in perm], slots=perm, split_tokens=-1)
    assert torch.equal(o, out[perm]) and torch.equal(l, lse[perm])
    o, l = p8.attend(lay, pool, q[3:4], [260], slots=[3], split_tokens=-1)
    assert torch.equal(o, out[3:4]) and torch.equal(l, lse[3:4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,H,G", [(128, 1, 4), (64, 8, 1), (32, 19, 2)])
def test_attend_pieces_of_long_prefixes(hd, H, G, dtype):
    lay = p8.Layout(1, 2, hd, 3001)
    lens = [3001, 0, 129, 1]
    pool, _, _ = filled(lay, lens, hide=0.3, seed=9)
    q = torch.randn((4, H, 2 * G, hd), generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
    for split, quota in [(0, 0), (128, 0), (1024, 0), (384, 0), (128, 3), (-1, 0), (0, 20)]:
        out, lse = p8.attend(lay, pool, q, lens, split_tokens=split, sm_quota=quota)
        check_attend(lay, pool, q, lens, out, lse, 0, 1 / math.sqrt(hd))
    a, b = p8.attend(lay, pool, q, lens, split_tokens=256), p8.attend(lay, pool, q, lens, split_tokens=256, sm_quota=7)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# calls that leave the SMs nearly empty share an item among 2, 4 or 8 warps, the long ones in pieces besides
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,kvh,hd,lens,hide", [
    (1, 1, 16, 64, [256], 0.0),                        # a tile for each of eight warps
    (1, 2, 2, 128, [33, 0, 1, 32, 31], 0.5),           # warps that get nothing, environments without tokens
    (19, 1, 2, 32, [700, 64, 0, 511], 0.9),            # warps that see nothing
    (8, 2, 16, 128, [640] * 6 + [7], 0.1),             # teams of four
    (32, 1, 16, 64, [2000] * 14, 0.0),                 # teams of two
    (5, 2, 1, 64, [9000, 20, 0, 8999], 0.3),           # pieces, each of a team
    (2, 1, 3, 128, [5000] + [3] * 40, 0.0),            # one long prefix among short ones
])
def test_attend_teams(H, G, kvh, hd, lens, hide, dtype):
    lay = p8.Layout(1, kvh, hd, max(lens))
    pool, _, _ = filled(lay, lens, hide=hide, seed=3)
    q = torch.randn((len(lens), H, kvh * G, hd), generator=torch.Generator().manual_seed(6)).to(DT[dtype]).cuda()
    out, lse = p8.attend(lay, pool, q, lens)
    check_attend(lay, pool, q, lens, out, lse, 0, 1 / math.sqrt(hd))
    again, _ = p8.attend(lay, pool, q, lens, out=q)
    assert torch.equal(again, out)


def test_attend_team_among_a_million_empty_items():
    lay = p8.Layout(1, 1, 32, 700)
    pool, _, _ = filled(lay, [700], seed=3)
    n, H, G = 1024, 1024, 9
    lens = [0] * (n - 1) + [700]
    q = torch.zeros((n, H, G, 32), dtype=torch.bfloat16, device="cuda")
    q[-1:] = torch.randn((1, H, G, 32), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    out, lse = p8.attend(lay, pool, q, lens, slots=[0] * n)
    assert (out[:-1] == 0).all() and torch.isneginf(lse[:-1]).all()
    check_attend(lay, pool, q[-1:], [700], out[-1:], lse[-1:], 0, 1 / math.sqrt(32))


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("split", [0, 128, 512, -1])
def test_attend_largest_values_and_what_one_piece_sees(hd, split):
    """Values near the end of fp32's range stay finite however they are cut; a NaN reaches who sees it, and nobody else."""
    P = 1500
    lay = p8.Layout(1, 1, hd, P)
    x = torch.randn((1, 1, 2, P, hd), generator=torch.Generator().manual_seed(2))
    x[:, :, 1] = 1e38 * torch.sign(x[:, :, 1])
    pool = p8.new_pool(lay, 1)
    p8.quantize(lay, pool, x.cuda(), [P])
    q = torch.randn((1, 4, 1, hd), generator=torch.Generator().manual_seed(6)).cuda()
    out, lse = p8.attend(lay, pool, q, [P], split_tokens=split)
    assert out.isfinite().all()
    check_attend(lay, pool, q, [P], out, lse, 0, 1 / math.sqrt(hd))
    x[0, 0, 1, 1400, 3] = float("nan")
    p8.quantize(lay, pool, x.cuda(), [P])
    assert p8.attend(lay, pool, q, [P], split_tokens=split)[0].isnan().all()
    o, l = p8.attend(lay, pool, q, [1376], split_tokens=split)
    check_attend(lay, pool, q, [1376], o, l, 0, 1 / math.sqrt(hd))


def test_attend_needs_a_workspace_for_pieces_only():
    dll = p8._load()
    for kvh, hd, H, G in ((1, 32, 1, 1), (16, 64, 1, 1), (4, 128, 32, 4)):
        for n in (1, 3, 200):
            for most, quota, needs in ((4096, 0, False), (256, 20, False), (70000, 0, n * kvh * H * G < 16 and kvh == 1)):
                lens = torch.full((n,), most, dtype=torch.int32)
                cl = p8._record(p8.Layout(1, kvh, hd, most))[2]
                need = dll.ebrl_prefix8_attend_workspace(cl, n, lens.data_ptr(), H, kvh * G, 0, quota)
                assert need > 0 if needs else (need == 0 or most > 4096), (kvh, hd, H, G, n, most, quota)
                assert need < 64 << 20
        lens = torch.ones(1000, dtype=torch.int32)          # the pieces of one long prefix cost the others no room
        lens[7] = 70000
        assert dll.ebrl_prefix8_attend_workspace(p8._record(p8.Layout(1, kvh, hd, 70000))[2], 1000, lens.data_ptr(), H, kvh * G, 0, 0) < 64 << 20


def test_attend_strided_queries_and_in_place():
    lay = p8.Layout(1, 2, 64, 90)
    lens = [90, 41, 7]
    pool, _, _ = filled(lay, lens)
    qkv = torch.randn((3, 8, 6, 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    q = qkv[:, :, 2:4]
    want, lse = p8.attend(lay, pool, q.contiguous(), lens)
    before = qkv.clone()
    out, _ = p8.attend(lay, pool, q, lens)
    assert torch.equal(out, want)
    wide = torch.full((3, 8, 6, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    p8.attend(lay, pool, q, lens, out=wide[:, :, 4:6])
    assert torch.equal(wide[:, :, 4:6], want) and (wide[:, :, :4] == 7).all()
    tok_major = torch.empty((8, 3, 2, 64), dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    p8.attend(lay, pool, q, lens, out=tok_major)
    assert torch.equal(tok_major, want)
    one = q[:, :1].expand(3, 8, 2, 64)                      # the same query for every token
    o, _ = p8.attend(lay, pool, one, lens)
    assert torch.equal(o, want[:, :1].expand(3, 8, 2, 64))
    p8.attend(lay, pool, q, lens, out=q)
    assert torch.equal(qkv[:, :, 2:4], want) and torch.equal(qkv[:, :, :2], before[:, :, :2]) and torch.equal(qkv[:, :, 4:], before[:, :, 4:])


def test_attend_records_beyond_32_bit_offsets():
    lay = p8.Layout(1, 4, 128, 4096)
    n_slots = 2 ** 32 // lay.record_bytes + 3
    pool = torch.empty((n_slots, lay.record_bytes), dtype=torch.uint8, device="cuda")
    assert pool.numel() > 2 ** 32
    slots, lens = [n_slots - 1, 0, n_slots // 2 + 1], [200, 64, 4096]
    planes = [planes_of(lay, P, "bf16", P).cuda() for P in lens]
    p8.quantize(lay, pool, planes, lens, slots=slots)
    q = torch.randn((3, 2, 4, 128), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()
    out, lse = p8.attend(lay, pool, q, lens, slots=slots)
    small = p8.new_pool(lay, 3)
    p8.quantize(lay, small, planes, lens)
    assert torch.equal(small, pool[slots])
    o, l = p8.attend(lay, small, q, lens)
    assert torch.equal(o, out) and torch.equal(l, lse)
    check_attend(lay, small, q, lens, out, lse, 0, 1 / math.sqrt(128))


def test_attend_more_environments_than_a_launch_takes():
    lay = p8.Layout(1, 1, 32, 33)
    n = 2500
    lens = [(i * 13) % 34 for i in range(n)]
    x = torch.randn((n, 1, 2, 33, 32), generator=torch.Generator().manual_seed(5)).cuda()
    pool = p8.new_pool(lay, n)
    p8.quantize(lay, pool, x, lens)
    q = torch.randn((n, 3, 1, 32), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    out, lse = p8.attend(lay, pool, q, lens)
    w = torch.zeros((n, 33), device="cuda")
    p8.weigh(lay, pool, q, lse, lens, w)
    for i in (0, 1, 1023, 1024, 1025, 2047, 2048, 2499):
        o, l = p8.attend(lay, pool, q[i:i + 1], [lens[i]], slots=[i])
        assert torch.equal(o[0], out[i]) and torch.equal(l[0], lse[i]), i
        assert abs(float(w[i].sum()) - (3 if lens[i] else 0)) < 1e-4
    check_attend(lay, pool[1020:1030], q[1020:1030], lens[1020:1030], out[1020:1030], lse[1020:1030], 0, 1 / math.sqrt(32))


# ---- weigh ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,kvh,hd,lens,cap,layers", SHAPES + [(2, 1, 16, 32, [500, 7], 500, 1), (4, 1, 9, 64, [1100], 1100, 1)])
def test_weigh_against_64_bits(H, G, kvh, hd, lens, cap, layers, dtype):
    lay = p8.Layout(layers, kvh, hd, cap)
    for hide, add in ((0.0, False), (0.5, True)):
        pool, _, _ = filled(lay, lens, hide=hide, seed=H + hd)
        n = len(lens)
        q = (1.5 * torch.randn((n, H, kvh * G, hd), generator=torch.Generator().manual_seed(H))).to(DT[dtype]).cuda()
        _, lse = p8.attend(lay, pool, q, lens, layer=layers - 1)
        if add:
            lse = lse.permute(2, 0, 1).contiguous().permute(1, 2, 0)     # heads outermost
        before = torch.rand((n, cap + 3), generator=torch.Generator().manual_seed(1)).cuda()
        for quota in (0, 2):
            w = before.clone()
            p8.weigh(lay, pool, q, lse, lens, w, layer=layers - 1, accumulate=add, sm_quota=quota)
            if quota:
                assert torch.equal(w, first)
            first = w
        for i in range(n):
            k, _, vis = decoded(lay, pool, i, layers - 1, lens[i])
            total, bound = np.zeros(lens[i]), 0.0
            for kh in range(kvh):
                ls = lse[i, :, kh * G:(kh + 1) * G].double().cpu().numpy().reshape(-1)
                if vis.any():
                    got, sa = ref.weigh(rows_of(q, i, kh, G), ls, k[kh], 1 / math.sqrt(hd))
                    total += got
                    bound = max(bound, 4 * hd * 2.0 ** -23 * sa + 2.0 ** -22 * (sa + np.abs(ls).max() + 2))
            total = np.where(vis, total, 0.0)
            base = before[i, :lens[i]].double().cpu().numpy() if add else 0.0
            tol = total * (bound + H * G * kvh * 2.0 ** -23) + 2.0 ** -23 * (base + total) + 1e-30
            assert (np.abs(w[i, :lens[i]].double().cpu().numpy() - base - total) <= tol).all(), i
            assert torch.equal(w[i, lens[i]:], before[i, lens[i]:])
            if vis.any() and not add:
                assert abs(float(w[i, :lens[i]].double().sum()) - H * G * kvh) < 1e-3 * H * G * kvh


# ---- evict ------------------------------------------------------------------------------------------------------------

def check_evict(lay, src, dst, dst0, weight, lens, keep, first, last, w_out, w_out0, kept, slots=None):
    codes, scales, words = (t.cpu().numpy() for t in p8.views(lay, src))
    c1, s1, m1 = (t.cpu().numpy() for t in p8.views(lay, dst))
    c0, s0, m0 = (t.cpu().numpy() for t in p8.views(lay, dst0))
    for i, n in enumerate(lens):
        sl = slots[i] if slots else i
        vis = [(int(words[sl, t // 32]) >> (t % 32)) & 1 for t in range(n)]
        idx = ref.select(weight[sl].cpu().numpy(), vis, n, keep[i], first, last)
        k, nb = len(idx), -(-len(idx) // 32)
        assert kept[i, :k].cpu().tolist() == idx, i
        assert [int(w) & 0xffffffff for w in m1[sl, :nb]] == [sum(vis[t] << b for b, t in enumerate(idx[32 * w:32 * w + 32])) for w in range(nb)]
        assert (m1[sl, nb:] == m0[sl, nb:]).all()
        if w_out is not None:
            assert torch.equal(w_out[sl, :k], weight[sl][idx]) or (w_out[sl, :k].isnan() == weight[sl][idx].isnan()).all()
            assert torch.equal(w_out[sl, k:], w_out0[sl, k:])
        for l in range(lay.kv_layers):
            for p in range(2):
                for h in range(lay.n_kv_heads):
                    x = ref.VALUES[codes[sl, l, p, h, idx]] * np.abs(scales[sl, l, p, h, [t // 32 for t in idx]]).astype(np.float64)[:, None] if k else np.zeros((0, lay.head_dim))
                    c, s = ref.quantize_head(x, np.ones(k, bool))
                    nan = np.isnan(ref.VALUES[c])
                    got = c1[sl, l, p, h, :k]
                    assert (np.where(nan, got & 127, got) == np.where(nan, 127, c)).all(), (i, l, p, h)
                    assert (s1[sl, l, p, h, :nb] == s.astype(np.float32)).all()
                    assert (c1[sl, l, p, h, k:] == c0[sl, l, p, h, k:]).all()
                    assert (s1[sl, l, p, h, nb:].view(np.int32) == s0[sl, l, p, h, nb:].view(np.int32)).all()


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_is_the_definition_bit_for_bit(hd, in_place):
    lay = p8.Layout(2, 2, hd, 700)
    lens = [700, 0, 1, 33, 64, 257, 511, 300, 512]
    keep = [350, 5, 1, 33, 0, 256, 300, 1000, 511]
    for hide, first, last in ((0.0, 0, 0), (0.4, 3, 20)):
        src, _, _ = filled(lay, lens, hide=hide, seed=hd)
        g = torch.Generator().manual_seed(hd)
        weight = torch.rand((len(lens), 705), generator=g)
        weight[0] = (weight[0] * 7).floor()                          # many ties
        weight[5] = 0.25                                             # nothing but ties
        weight[6, ::3] = -weight[6, ::3]
        weight[6, 1], weight[6, 2], weight[6, 5], weight[6, 8], weight[6, 11] = math.nan, math.inf, -math.inf, -0.0, 0.0
        weight = weight.cuda()
        src0, w0 = src.clone(), weight.clone()
        dst = src if in_place else torch.full_like(src, 0x33)
        dst0 = dst.clone()
        w_out = weight if in_place else torch.full_like(weight, 9.0)
        w_out0 = w_out.clone()
        new, kept = p8.evict(lay, src, dst, weight, lens, keep, protect_first=first, protect_last=last, weight_out=w_out)
        assert new.tolist() == [min(a, b) for a, b in zip(lens, keep)]
        check_evict(lay, src0, dst, dst0, w0, lens, keep, first, last, w_out, w_out0, kept)


def test_evict_slots_quota_kept_buffer_and_more_environments_than_a_launch_takes():
    lay = p8.Layout(1, 1, 32, 50)
    n = 600
    lens = [(i * 17) % 51 for i in range(n)]
    keep = [(i * 5) % 40 for i in range(n)]
    x = torch.randn((n, 1, 2, 50, 32), generator=torch.Generator().manual_seed(5)).cuda()
    src = p8.new_pool(lay, n + 10)
    slots = (torch.randperm(n + 10, generator=torch.Generator().manual_seed(2))[:n]).tolist()
    p8.quantize(lay, src, x, lens, slots=slots)
    weight = torch.rand((n + 10, 50), generator=torch.Generator().manual_seed(3)).cuda()
    res = []
    for quota in (0, 3):
        dst = torch.full_like(src, 0x22)
        kept = torch.full((n, 44), -5, dtype=torch.int32, device="cuda")
        p8.evict(lay, src, dst, weight, lens, keep, slots=slots, kept=kept, sm_quota=quota)
        res.append((dst, kept))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    dst, kept = res[0]
    check_evict(lay, src, dst, torch.full_like(src, 0x22), weight, lens, keep, 0, 0, None, None, kept, slots=slots)
    for i in (0, 7, 511, 512, 599):
        assert (kept[i, min(lens[i], keep[i]):] == -5).all()


def test_evict_long_prefix_in_many_chunks():
    lay = p8.Layout(1, 1, 128, 20000)
    lens, keep = [20000, 17], [7777, 16]
    src, _, _ = filled(lay, lens, seed=2)
    weight = torch.rand((2, 20000), generator=torch.Generator().manual_seed(3)).cuda()
    weight[0, ::2] = weight[0, 1::2]
    dst = torch.full_like(src, 0x22)
    dst0 = dst.clone()
    _, kept = p8.evict(lay, src, dst, weight, lens, keep)
    check_evict(lay, src, dst, dst0, weight, lens, keep, 0, 0, None, None, kept)
    again = src.clone()
    _, kept2 = p8.evict(lay, again, again, weight, lens, keep)
    a, b = p8.views(lay, again), p8.views(lay, dst)
    assert torch.equal(kept[0], kept2[0]) and torch.equal(kept[1, :16], kept2[1, :16])
    assert torch.equal(a[0][0, ..., :7777, :], b[0][0, ..., :7777, :]) and torch.equal(a[1][0, ..., :244], b[1][0, ..., :244])


# ---- together, streams, graphs ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,hd,H", [("bf16", 128, 16), ("f32", 64, 8)])
def test_write_read_weigh_shorten_read(dtype, hd, H):
    """The life of a cache: written, attended to over two Euler steps while the weights add up, halved in place, attended to again."""
    lay = p8.Layout(2, 4, hd, 300)
    lens = [300, 120, 33, 64]
    pool, _, _ = filled(lay, lens, dtype=dtype, hide=0.1, seed=1)
    weight = torch.zeros((4, 300), device="cuda")
    scale = 1 / math.sqrt(hd)
    for step in range(2):
        for layer in range(2):
            q = torch.randn((4, H, 4, hd), generator=torch.Generator().manual_seed(10 * step + layer)).to(DT[dtype]).cuda()
            out, lse = p8.attend(lay, pool, q, lens, layer=layer)
            check_attend(lay, pool, q, lens, out, lse, layer, scale)
            p8.weigh(lay, pool, q, lse, lens, weight, layer=layer)
    for i in range(4):
        assert abs(float(weight[i].sum()) - (4 * H * 4 if i != 2 else 0)) < 0.01 * 4 * H * 4   # environment 2 sees nothing
    before = pool.clone()
    new, kept = p8.evict(lay, pool, pool, weight, lens, [l // 2 for l in lens], protect_last=4, weight_out=weight)
    assert new.tolist() == [150, 60, 16, 32]
    q = torch.randn((4, H, 4, hd), generator=torch.Generator().manual_seed(77)).to(DT[dtype]).cuda()
    out, lse = p8.attend(lay, pool, q, new, layer=1)
    check_attend(lay, pool, q, new.tolist(), out, lse, 1, scale)
    # and what is left is what was kept: powers of two move no bits unless a code falls below the new block's smallest
    for i in range(4):
        k0, v0, vis0 = decoded(lay, before, i, 0, lens[i])
        k1, v1, vis1 = decoded(lay, pool, i, 0, int(new[i]))
        idx = kept[i, :int(new[i])].cpu().numpy()
        _, sc, _ = p8.views(lay, pool)
        for a, b, plane in ((k0, k1, 0), (v0, v1, 1)):
            fine = np.repeat(sc[i, 0, plane].double().cpu().numpy(), 32, axis=-1)[:, :int(new[i]), None] * 2.0 ** -10
            assert (np.abs(a[:, idx] - b) <= fine).all()
        assert (vis0[idx] == vis1).all()


def test_operators_on_another_stream_and_captured():
    lay = p8.Layout(1, 2, 64, 1500)
    lens = [1500, 700]
    planes = [planes_of(lay, P, "bf16", P).cuda() for P in lens]
    q = torch.randn((2, 1, 4, 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()

    def chain(stream=None):
        pool = p8.new_pool(lay, 2)
        w = torch.zeros((2, 1500), device="cuda")
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        p8.quantize(lay, pool, planes, lens, stream=stream)
        out, lse = p8.attend(lay, pool, q, lens, split_tokens=256, stream=stream)
        p8.weigh(lay, pool, q, lse, lens, w, stream=stream)
        new, kept = p8.evict(lay, pool, pool, w, lens, 500, stream=stream)
        return pool, out, lse, w, kept

    want = chain()
    s = torch.cuda.Stream()
    got = chain(s)
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    # captured twice (two graphs, each with its own workspace), replayed in turn and on new queries
    graphs = []
    for _ in range(2):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = chain()
        graphs.append((g, res))
    for g, _ in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    for _, res in graphs:
        for a, b in zip(res, want):
            assert torch.equal(a, b)
    q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16))
    graphs[0][0].replay()
    again = chain()
    torch.cuda.synchronize()
    for a, b in zip(graphs[0][1], again):
        assert torch.equal(a, b)


def test_two_calls_at_once():
    """Long prefixes (own workspaces) on two streams."""
    lay = p8.Layout(1, 2, 64, 4000)
    pool, _, _ = filled(lay, [4000, 3000])
    qs = [torch.randn((2, 1, 4, 64), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).cuda() for i in range(2)]
    want = [p8.attend(lay, pool, q, [4000, 3000], split_tokens=128) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(20):
        got = [p8.attend(lay, pool, q, [4000, 3000], split_tokens=128, stream=s) for q, s in zip(qs, streams)]
    torch.cuda.synchronize()
    for (a, b), (c, d) in zip(got, want):
        assert torch.equal(a, c) and torch.equal(b, d)
