"""GPU tests of the operators on 8-bit prefix records at their limits: the smallest and the largest scales, calls without
query rows, rows of a single environment or token, score-sized sums whose difference is small, how a call is launched."""
import concurrent.futures
import ctypes as C
import math

import numpy as np
import pytest
import torch

import prefix8_reference as ref
from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import prefix8 as p8
from test_prefix8_gpu import DT, check_attend, check_evict, decoded, filled, planes_of, rows_of
from test_prefix8_handle_gpu import Case

pytestmark = pytest.mark.gpu


class _Edge(C.Structure):
    _fields_ = [("from_port", C.c_ubyte), ("to_port", C.c_ubyte), ("type", C.c_ubyte), ("reserved", C.c_ubyte * 5)]


def captured(call):
    """A captured call's graph (kept)."""
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call()
    return g


def edge_types(g):
    """The types of a graph's edges: 0 = full, 1 = programmatic (the later kernel may be resident before the earlier one is done)."""
    cu = C.CDLL("libcuda.so.1")
    n = C.c_size_t(0)
    raw = C.c_void_p(g.raw_cuda_graph())
    assert cu.cuGraphGetEdges_v2(raw, None, None, None, C.byref(n)) == 0
    a, b, e = (C.c_void_p * n.value)(), (C.c_void_p * n.value)(), (_Edge * n.value)()
    assert cu.cuGraphGetEdges_v2(raw, a, b, e, C.byref(n)) == 0
    return [x.type for x in e]


# ---- how a call is launched -------------------------------------------------------------------------------------------

def test_the_join_is_not_resident_early_under_a_quota():
    """Under a quota the join's CTAs must not wait on SMs beside the attention's own: the launch is an ordinary one."""
    lay = p8.Layout(1, 2, 64, 1500)
    pool, _, _ = filled(lay, [1500, 700])
    q = torch.randn((2, 1, 4, 64), generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda()

    def call(quota):
        return lambda: p8.attend(lay, pool, q, [1500, 700], split_tokens=256, sm_quota=quota)
    call(0)(), call(8)()
    assert edge_types(captured(call(0))) == [1]
    assert edge_types(captured(call(8))) == [0]
    assert edge_types(captured(call(0))) == [1]


class _Kernel(C.Structure):
    _fields_ = [("func", C.c_void_p), ("grid", C.c_uint * 3), ("block", C.c_uint * 3), ("shared", C.c_uint), ("params", C.c_void_p), ("extra", C.c_void_p),
                ("kern", C.c_void_p), ("ctx", C.c_void_p)]


def warps_of(g):
    """Warps per CTA of a graph's kernels, in ascending order."""
    cu = C.CDLL("libcuda.so.1")
    n = C.c_size_t(0)
    raw = C.c_void_p(g.raw_cuda_graph())
    assert cu.cuGraphGetNodes(raw, None, C.byref(n)) == 0
    nodes = (C.c_void_p * n.value)()
    assert cu.cuGraphGetNodes(raw, nodes, C.byref(n)) == 0
    out = []
    for node in nodes:
        k = _Kernel()
        assert cu.cuGraphKernelNodeGetParams_v2(C.c_void_p(node), C.byref(k)) == 0
        out.append(k.block[0] // 32)
    return sorted(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,kvh,hd,lens,want", [
    (1, 1, 16, 64, [256], [8]),                         # a tile for each of eight warps
    (1, 2, 2, 128, [33, 0, 1, 32, 31], [2]),            # two tiles at most
    (19, 1, 2, 32, [700, 64, 0, 511], [8]),
    (8, 2, 16, 128, [640] * 6 + [7], [4]),
    (32, 1, 16, 64, [2000] * 14, [2]),
    (5, 2, 1, 64, [9000, 20, 0, 8999], [4, 16]),        # pieces, each of a team, and their join
    (2, 1, 3, 128, [5000] + [3] * 40, [4, 16]),
    (8, 1, 16, 64, [256] * 200, [1]),                   # the SMs are full
])
def test_which_form_a_call_takes(H, G, kvh, hd, lens, want, dtype):
    """The calls that test teams, pieces and both really run them (on 148 SMs)."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the choice goes by the number of SMs")
    lay = p8.Layout(1, kvh, hd, max(lens))
    pool = p8.new_pool(lay, len(lens))
    q = torch.zeros((len(lens), H, kvh * G, hd), dtype=DT[dtype], device="cuda")
    p8.attend(lay, pool, q, lens)
    assert warps_of(captured(lambda: p8.attend(lay, pool, q, lens))) == want


# ---- scales -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("split", [-1, 0, 128])
def test_attend_subnormal_scales(dtype, split):
    """A caller's scales may lie below the smallest normal number, in the first block that a row sees, too."""
    lay = p8.Layout(1, 1, 64, 300)
    pool, _, _ = filled(lay, [300], seed=4, poison=False)
    _, scales, _ = p8.views(lay, pool)
    kept = scales.clone()
    q = torch.randn((1, 8, 1, 64), generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
    for at in (0, 1, 9, slice(0, 4), slice(0, 10)):
        for small in (2.0 ** -127, 1e-39, 1e-40, 1e-45):
            scales.copy_(kept)
            scales[0, 0, 1, 0, at] = small
            out, lse = p8.attend(lay, pool, q, [300], split_tokens=split)
            check_attend(lay, pool, q, [300], out, lse, 0, 1 / 8)
    scales.copy_(kept)
    scales[0, 0, 0, 0, 0] = 1e-40
    out, lse = p8.attend(lay, pool, q, [300], split_tokens=split)
    check_attend(lay, pool, q, [300], out, lse, 0, 1 / 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("P,split", [(40, -1), (1500, -1), (1500, 0), (1500, 128), (6000, 0)])
def test_attend_small_values_keep_their_bits(P, split, hd, dtype):
    """Values 2^-118 times as large give outputs 2^-118 times as large, bit for bit where those are normal numbers: nothing
    on the way (the unit of the sums divided by the sum of the weights, say) may fall below what fp32 holds with 24 bits.

    Of prefixes that are cut into n pieces, the pieces' means and the sums that join them may fall below 2^-126 where the
    output does not: rounded to multiples of 2^-149, off by 2^-32 of the large values' unit instead of 2^-24 of themselves.  The
    factors f of the means are the same in both calls (lse is), and sum to 1.  So the two joins' sums drift apart by f 2^-32 (the mean) +
    2^-32 + 2 x 2^-24 A (the roundings of either sum, of size A at most) at every piece: 2^-32 (n + 1) + n 2^-23 A in all, and
    a bf16 output may round the other way (2^-8)."""
    lay = p8.Layout(1, 2, hd, P)
    x = torch.randn((1, 1, 2, P, 2 * hd), generator=torch.Generator().manual_seed(P))
    q = torch.randn((1, 8, 2, hd), generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
    pool = p8.new_pool(lay, 1)
    p8.quantize(lay, pool, x.cuda(), [P])
    want, lse = p8.attend(lay, pool, q, [P], split_tokens=split)
    x[:, :, 1] *= 2.0 ** -118
    p8.quantize(lay, pool, x.cuda(), [P])
    _, scales, _ = p8.views(lay, pool)
    assert float(scales[0, 0, 1, :, :-(-P // 32)].max()) <= 2.0 ** -123   # (and 2^-126 at least: none was bounded)
    out, lse2 = p8.attend(lay, pool, q, [P], split_tokens=split)
    assert torch.equal(lse, lse2)
    normal = want.float().abs() >= 2.0 ** -7
    assert normal.any()
    got, want = out.float() * 2.0 ** 118, want.float()
    if split == -1 or (split == 0 and P <= 4096):         # not cut
        assert torch.equal(got[normal], want[normal])
        return
    n = -(-P // (split or 512))                           # (left to itself no piece is shorter than 512 tokens)
    p8.quantize(lay, pool, (x * torch.tensor([1.0, 2.0 ** 118])[None, None, :, None, None]).cuda(), [P])
    k, v, _ = decoded(lay, pool, 0, 0, P)
    for kh in range(2):
        s = rows_of(q, 0, kh, 1) @ k[kh].T / math.sqrt(hd)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        A = np.zeros((8, hd))                             # the largest partial sum, wherever the cuts are (they lie between tiles)
        part = np.zeros((8, hd))
        for t in range(0, P, 32):
            part = part + w[:, t:t + 32] @ v[kh, t:t + 32]
            A = np.maximum(A, np.abs(part))
        tol = 1.001 * (2.0 ** -32 * (n + 1) + n * 2.0 ** -23 * A)
        a, b = rows_of(got, 0, kh, 1), rows_of(want, 0, kh, 1)
        ok = np.abs(a - b) <= tol + (np.abs(b) * 2.0 ** -8 if dtype == "bf16" else 0.0)
        assert ok[rows_of(normal, 0, kh, 1) != 0].all()


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_largest_values(hd, in_place):
    """A code times its scale may pass fp32's largest number (3.35e38 is kept as 256 x 2^120): the new block's scale goes by it all the same."""
    lay = p8.Layout(1, 2, hd, 400)
    lens, keep = [400, 400, 64], [200, 40, 40]
    x = [planes_of(lay, P, "f32", P) for P in lens]
    x[0][0, :, 3, 1], x[0][0, 1, 100, 2], x[0][0, 0, 390, hd + 5] = 3.35e38, -3.4e38, 3.3e38
    x[1][0, :, 40, 0] = -3.4e38
    src = p8.new_pool(lay, 3)
    p8.quantize(lay, src, [t.cuda() for t in x], lens)
    _, scales, _ = p8.views(lay, src)
    assert float(scales[0, 0, 0, 0, 0]) == 2.0 ** 120
    scales[1] *= 1.25                                     # not a power of two
    scales[2, 0, :, 0, 0] = 2.0 ** 127                    # the largest power of two, whatever the codes
    weight = torch.rand((3, 400), generator=torch.Generator().manual_seed(3)).cuda()
    weight[:, 3] = weight[:, 40] = weight[:, 100] = 2.0
    weight[0, 390] = 2.0
    src0, dst = src.clone(), src if in_place else torch.full_like(src, 0x33)
    dst0 = dst.clone()
    _, kept = p8.evict(lay, src, dst, weight, lens, keep)
    check_evict(lay, src0, dst, dst0, weight, lens, keep, 0, 0, None, None, kept)


# ---- weigh ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("H,heads", [(0, 2), (3, 0), (0, 0)])
def test_weigh_without_query_rows(H, heads):
    """The sum over no rows is 0: written where the call writes, added where it adds; the rest of the row stays."""
    lay = p8.Layout(1, 2, 64, 90)
    lens, slots = [90, 0, 40], [3, 0, 1]
    pool, _, _ = filled(lay, lens, slots=slots, n_slots=4, hide=0.3)
    q, lse = torch.empty((3, H, heads, 64), device="cuda"), torch.empty((3, H, heads), device="cuda")
    w = torch.full((4, 95), 5.0, device="cuda")
    assert p8.weigh(lay, pool, q, lse, lens, w, slots=slots) is w
    assert (w == 5).all()
    for quota in (0, 2):
        w.fill_(5.0)
        p8.weigh(lay, pool, q, lse, lens, w, slots=slots, accumulate=False, sm_quota=quota)
        want = torch.full((4, 95), 5.0, device="cuda")
        want[3, :90], want[1, :40] = 0.0, 0.0
        assert torch.equal(w, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,H", [(32, 3), (64, 8), (128, 8), (128, 16), (64, 33)])
def test_weigh_differences_of_large_scores(hd, H, dtype):
    """Scores of hundreds next to a log-sum-exp as large.  One column of keys and queries is not zero and everything in it has few
    bits, so a score is exact; what is left is the difference a = score - lse (rounded: 2^-24 of it), a in units of log 2 (2^-24 for the
    product, 2^-25 for the constant), the power (2^-22) and the sum over the rows (2^-24 each)."""
    P = 200
    lay = p8.Layout(1, 1, hd, P)
    g = torch.Generator().manual_seed(hd + H)
    x = torch.zeros((1, 1, 2, P, hd))
    x[0, 0, 0, :, 5] = torch.randint(32, 38, (P,), generator=g).float()          # kept as 32 or 36
    pool = p8.new_pool(lay, 1)
    p8.quantize(lay, pool, x.cuda(), [P])
    q = torch.zeros((1, H, 1, hd))
    q[0, :, 0, 5] = torch.randint(30, 60, (H,), generator=g).float()
    scale = 0.123
    k, _, _ = decoded(lay, pool, 0, 0, P)
    s = float(np.float32(scale)) * (rows_of(q, 0, 0, 1) @ k[0].T)                # [H, P] in 64 bits
    # (rows whose difference is far from 0 add nothing that counts)
    lse = torch.from_numpy(np.median(s, axis=1)).float().view(1, H, 1) + torch.rand((1, H, 1), generator=g)
    a = s - lse[0].double().numpy()
    p = np.exp(a)
    want = p.sum(0)
    tol = (p * (np.abs(a) * (2.0 ** -24 + 2.0 ** -24 + 2.0 ** -25) + 2.0 ** -22 + H * 2.0 ** -24)).sum(0) + 1e-37
    w = torch.zeros((1, P), device="cuda")
    p8.weigh(lay, pool, q.to(DT[dtype]).cuda(), lse.cuda(), [P], w, scale=scale, accumulate=False)
    err = np.abs(w[0].double().cpu().numpy() - want)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("H", [2, 16, 40])
def test_weigh_second_terms_of_fp32_queries(H, hd):
    """Queries of more bits than one f16 term holds, in every 16 columns that are contracted at a time.  The first terms' products add up to
    whole numbers below 2^24 (exact), the second terms' are 0.75 each: a sum that loses a fraction at every step would be off by up to hd / 16
    units of 1.3e7, which scores of hundreds show.  The total is a whole number again, so scores are exact; the tolerance is that of the test above."""
    P = 200
    lay = p8.Layout(1, 1, hd, P)
    g = torch.Generator().manual_seed(hd + H)
    cols = [4 * st for st in range(hd // 16)]                                    # one in every step
    x, q = torch.zeros((1, 1, 2, P, hd)), torch.zeros((1, H, 1, hd))
    x[0, 0, 0, :, cols] = 1.0
    x[0, 0, 0, :, 1] = torch.where(torch.rand(P, generator=g) < 0.5, 448.0, 416.0)
    x[0, 0, 0, ::32, 1] = 448.0                                                  # (every block's scale is 1)
    q[0, :, 0, cols] = 4096.75
    if len(cols) % 4:
        q[0, :, 0, cols[0]] = 4096.5                                             # 0.5 + 0.5 are whole, too
        q[0, :, 0, cols[1]] = 4096.5
    q[0, :, 0, 1] = torch.where(torch.rand(H, generator=g) < 0.5, 28672.0, 26624.0)
    scale = float(np.float32(1.7e-5))
    pool = p8.new_pool(lay, 1)
    p8.quantize(lay, pool, x.cuda(), [P])
    k, _, _ = decoded(lay, pool, 0, 0, P)
    s = rows_of(q, 0, 0, 1) @ k[0].T
    assert (s == np.rint(s)).all() and s.max() < 2 ** 24 and s.min() > 2 ** 23
    s = scale * s
    lse = torch.from_numpy(s.max(1)).float().view(1, H, 1) + torch.rand((1, H, 1), generator=g)
    a = s - lse[0].double().numpy()
    p = np.exp(a)
    tol = (p * (np.abs(a) * (2.0 ** -24 + 2.0 ** -24 + 2.0 ** -25) + 2.0 ** -22 + H * 2.0 ** -24)).sum(0) + 1e-37
    w = torch.zeros((1, P), device="cuda")
    p8.weigh(lay, pool, q.cuda(), lse.cuda(), [P], w, scale=scale, accumulate=False)
    err = np.abs(w[0].double().cpu().numpy() - p.sum(0))
    assert (err <= tol).all(), float((err / tol).max())


# ---- strides ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_of_a_single_environment_or_token_do_not_matter(dtype):
    lay = p8.Layout(1, 2, 64, 90)
    pool, _, _ = filled(lay, [90, 41], seed=2)
    flat = torch.randn(4000, generator=torch.Generator().manual_seed(5)).to(DT[dtype]).cuda()
    w = torch.zeros((2, 90), device="cuda")

    def both(q, lens):
        want, lse = p8.attend(lay, pool, q.contiguous(), lens)
        got, l2 = p8.attend(lay, pool, q, lens)
        assert torch.equal(got, want) and torch.equal(l2, lse)
        into = torch.empty(2000, dtype=q.dtype, device="cuda").as_strided(q.shape, q.stride())
        p8.attend(lay, pool, q, lens, out=into)
        assert torch.equal(into, want)
        a = p8.weigh(lay, pool, q, lse, lens, w.clone())
        assert torch.equal(a, p8.weigh(lay, pool, q.contiguous(), lse, lens, w.clone()))
    both(flat.as_strided((1, 3, 2, 64), (3, 128, 64, 1)), [90])
    both(flat.as_strided((2, 1, 2, 64), (256, 7, 64, 1)), [90, 41])
    both(flat.as_strided((1, 1, 2, 64), (5, 3, 64, 1)), [90])


def test_evict_weights_next_to_one_another():
    """The weights before and after in one tensor, row by row."""
    lay = p8.Layout(1, 2, 32, 100)
    lens, keep = [100, 33, 64], [50, 33, 7]
    src, _, _ = filled(lay, lens, seed=2)
    both = torch.rand((3, 2, 100), generator=torch.Generator().manual_seed(3)).cuda()
    for a, b in ((0, 1), (1, 0)):
        w0, dst = both.clone(), torch.full_like(src, 0x33)
        _, kept = p8.evict(lay, src, dst, both[:, a], lens, keep, weight_out=both[:, b])
        check_evict(lay, src, dst, torch.full_like(src, 0x33), w0[:, a], lens, keep, 0, 0, both[:, b], w0[:, b], kept)
        assert torch.equal(both[:, a], w0[:, a])
        for i in range(3):
            k = min(lens[i], keep[i])
            assert torch.equal(both[i, b, :k], w0[i, a, kept[i, :k].long()])


# ---- evict beyond what selection keeps in shared memory ---------------------------------------------------------------

@pytest.mark.parametrize("in_place", [False, True])
def test_evict_prefixes_of_any_length_in_one_call(in_place):
    """Selection holds the keys of up to 49152 tokens in shared memory and makes them anew from the weights beyond: both, at the border, in
    one call, with ties, hidden tokens and protected ends."""
    lay = p8.Layout(1, 1, 32, 70000)
    lens = [49152, 49153, 70000, 50, 70000, 60000, 0]
    keep = [20000, 20000, 35000, 20, 70000, 1, 5]
    src, _, _ = filled(lay, lens, hide=0.3, seed=5)
    weight = torch.rand((len(lens), 70000), generator=torch.Generator().manual_seed(3))
    weight[1, 10::3] = 0.5
    weight[2] = (weight[2] * 5).floor()                   # the last kept key is a tie among thousands
    weight[4, ::7], weight[5] = math.nan, -0.0
    weight = weight.cuda()
    src0, w0 = src.clone(), weight.clone()
    dst = src if in_place else torch.full_like(src, 0x33)
    dst0 = dst.clone()
    w_out = weight if in_place else torch.full_like(weight, 9.0)
    w_out0 = w_out.clone()
    _, kept = p8.evict(lay, src, dst, weight, lens, keep, protect_first=3, protect_last=40, weight_out=w_out)
    check_evict(lay, src0, dst, dst0, w0, lens, keep, 3, 40, w_out, w_out0, kept)
    for i, (n, k) in enumerate(zip(lens, keep)):
        k = min(n, k)
        assert torch.equal(w_out[i, :k].view(torch.int32), w0[i, kept[i, :k].long()].view(torch.int32)), i


# ---- what evict writes beside the records -----------------------------------------------------------------------------

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("quota", [0, 3])
def test_evict_weights_bit_for_bit(in_place, quota):
    """The kept tokens' weights, NaN and signed zeros among them, by slot, in place and under a quota."""
    lay = p8.Layout(2, 2, 64, 300)
    lens, keep, slots = [300, 0, 33, 257, 64], [150, 4, 33, 99, 0], [5, 1, 0, 3, 4]
    src, _, _ = filled(lay, lens, hide=0.2, seed=1, n_slots=6, slots=slots)
    weight = torch.randn((6, 301), generator=torch.Generator().manual_seed(3)).cuda()
    weight[5, ::4], weight[3, ::5], weight[3, 1::5] = math.nan, -0.0, 0.0
    src0, w0 = src.clone(), weight.clone()
    dst = src if in_place else torch.full_like(src, 0x33)
    dst0 = dst.clone()
    w_out = weight if in_place else torch.full_like(weight, 9.0)
    w_out0 = w_out.clone()
    _, kept = p8.evict(lay, src, dst, weight, lens, keep, slots=slots, protect_first=2, weight_out=w_out, sm_quota=quota)
    check_evict(lay, src0, dst, dst0, w0, lens, keep, 2, 0, None, None, kept, slots=slots)
    want = w_out0.clone()
    for i, sl in enumerate(slots):
        k = min(lens[i], keep[i])
        want[sl, :k] = w0[sl, kept[i, :k].long()]
    assert torch.equal(w_out.view(torch.int32), want.view(torch.int32))


# ---- more environments than a launch takes ----------------------------------------------------------------------------

def test_quantize_slots_masks_and_strides_across_launches():
    lay = p8.Layout(1, 2, 32, 40)
    n = 2300
    x = torch.randn((n, 1, 2, 48, 128), generator=torch.Generator().manual_seed(1)).cuda()[:, :, :, :40, 32:96]
    lens = [(7 * i) % 41 for i in range(n)]
    g = torch.Generator().manual_seed(2)
    slots = torch.randperm(n + 20, generator=g)[:n].to(torch.int32)
    mask = (torch.rand((n, 40), generator=g) > 0.3).cuda()
    a = p8.new_pool(lay, n + 20)
    a.fill_(0x55)
    p8.quantize(lay, a, x, lens, slots=slots, mask=mask)
    b = torch.full_like(a, 0x55)
    for i in range(0, n, 500):                            # one launch each
        j = min(n, i + 500)
        p8.quantize(lay, b, [x[k, :, :, :lens[k]].contiguous() for k in range(i, j)], lens[i:j], slots=slots[i:j], mask=[mask[k] for k in range(i, j)])
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("quota", [0, 5])
def test_attend_pieces_of_more_environments_than_a_launch_takes(dtype, quota):
    lay = p8.Layout(1, 1, 32, 300)
    n = 1100
    lens = [(i * 37) % 301 for i in range(n)]
    x = torch.randn((n, 1, 2, 300, 32), generator=torch.Generator().manual_seed(5)).cuda()
    pool = p8.new_pool(lay, n)
    p8.quantize(lay, pool, x, lens)
    q = torch.randn((n, 3, 2, 32), generator=torch.Generator().manual_seed(6)).to(DT[dtype]).cuda()
    out, lse = p8.attend(lay, pool, q, lens, split_tokens=128, sm_quota=quota)
    o, l = p8.attend(lay, pool, q, lens, split_tokens=-1)
    for i in list(range(1018, 1030)) + [0, 1, n - 1]:
        check_attend(lay, pool[i:i + 1], q[i:i + 1], lens[i:i + 1], out[i:i + 1], lse[i:i + 1], 0, 1 / math.sqrt(32))
    # all others against the uncut call: the scores' bits are the same, sums of up to 300 weights are off by (300 / 8 + 64) 2^-24 on either
    # side, lse (below 15) by 2^-22 (1 + lse) besides, weights by 2^-11, outputs by 2^-8 of themselves
    sums, vmax = (300 / 8 + 64) * 2.0 ** -24, float(x[:, :, 1].abs().max()) * 1.07
    assert torch.equal(torch.isneginf(l), torch.isneginf(lse)) and float(lse.max()) < 15
    assert float((l - lse).nan_to_num(0.0).abs().max()) <= 2 * (sums + 2.0 ** -22 * 16)
    assert ((o.float() - out.float()).abs() <= 2.0 ** -7 * o.float().abs() + 2 * (2 * sums + 2.0 ** -11) * vmax).all()


def test_attend_teams_in_more_than_one_launch():
    """Few environments with tokens among many without: a team for each of them, and a launch that has none."""
    lay = p8.Layout(1, 2, 64, 800)
    n = 2100
    pool, _, _ = filled(lay, [800, 513, 64], seed=3)
    lens, slots = [0] * n, [0] * n
    for i, (at, ln) in enumerate(((3, 800), (1023, 513), (2099, 64))):
        lens[at], slots[at] = ln, i
    q = torch.randn((n, 2, 2, 64), generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    out, lse = p8.attend(lay, pool, q, lens, slots=slots)
    at = [3, 1023, 2099]
    check_attend(lay, pool, q[at], [800, 513, 64], out[at], lse[at], 0, 1 / 8)
    rest = torch.ones(n, dtype=torch.bool)
    rest[at] = False
    assert (out[rest.cuda()] == 0).all() and torch.isneginf(lse[rest.cuda()]).all()


# ---- several host threads ---------------------------------------------------------------------------------------------

def test_calls_from_several_threads():
    """Four threads, each with its own stream, pool and weights: every result is that of the same calls one after another."""
    lay = p8.Layout(1, 2, 64, 700)
    sets = []
    for i in range(4):
        lens = [700 - 100 * i, 33 + i, 64]
        planes = [planes_of(lay, P, "bf16", P + i).cuda() for P in lens]
        q = torch.randn((3, 4, 2, 64), generator=torch.Generator().manual_seed(i)).to(torch.bfloat16 if i % 2 else torch.float32).cuda()
        sets.append((lens, planes, q, torch.cuda.Stream()))

    def life(lens, planes, q, stream):
        with torch.cuda.stream(stream):
            pool, w = p8.new_pool(lay, 3), torch.zeros((3, 700), device="cuda")
            p8.quantize(lay, pool, planes, lens)
            for split in (-1, 128, 0):
                out, lse = p8.attend(lay, pool, q, lens, split_tokens=split)
            p8.weigh(lay, pool, q, lse, lens, w)
            _, kept = p8.evict(lay, pool, pool, w, lens, [n // 2 for n in lens], kept=torch.zeros((3, 700), dtype=torch.int32, device="cuda"))
            with pytest.raises(p8.EbrlError, match="layer 7"):
                p8.attend(lay, pool, q, lens, layer=7)
            stream.synchronize()
        return pool, out, lse, w, kept
    torch.cuda.synchronize()
    want = [life(*s) for s in sets]
    for _ in range(5):
        with concurrent.futures.ThreadPoolExecutor(4) as ex:
            got = list(ex.map(lambda s: life(*s), sets))
        for a, b in zip(got, want):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


# ---- handles ----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_handle_environments_that_see_nothing(dtype):
    """All tokens hidden: cross-attention gives 0, as it does over values of 0, and no token gets any weight."""
    c = Case(dtype=dtype, P=(5, 90))
    none = [2, 7]
    gen = B.ActGen(c.cfg, c.wt)
    w = torch.zeros((12, c.cfg.max_prefix_len), device="cuda")
    zero = torch.zeros((1, 2, 90, 256), dtype=DT[dtype], device="cuda")
    base = c.run(gen, [list(range(12))])
    p8.quantize(c.lay, c.pool, [zero[:, :, :c.P[i]].contiguous() for i in none], [c.P[i] for i in none], slots=none)
    want = c.run(gen, [list(range(12))])
    planes = [torch.full((1, 2, c.P[i], 256), math.nan, dtype=DT[dtype], device="cuda") for i in none]
    p8.quantize(c.lay, c.pool, planes, [c.P[i] for i in none], slots=none, mask=[torch.zeros(c.P[i], dtype=torch.uint8, device="cuda") for i in none])
    got = c.run(gen, [list(range(12))], weights=w)
    gen.destroy()
    rest = [i for i in range(12) if i not in none]
    assert np.array_equal(got, want) and np.array_equal(got[rest], base[rest]) and not np.array_equal(got[none], base[none])
    assert (w[none] == 0).all() and (w[rest].sum(1) > 0).all()
