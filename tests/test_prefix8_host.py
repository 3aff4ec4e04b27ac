"""CPU-only tests of the 8-bit prefix cache operators: the record's layout, every refusal (arguments are checked before
anything touches a device) and the handle's configuration rules."""
import ctypes as C

import numpy as np
import pytest
import torch

import prefix8_reference as ref
from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import prefix8 as p8

L = p8._load()
LAY = p8.Layout(2, 4, 64, 100)
P0 = 0x10000     # an aligned address that is never touched


def lay(**kw):
    return C.byref(p8._CLayout(*LAY._replace(**kw)))


def ints(v):
    return None if v is None else (C.c_int32 * max(1, len(v)))(*v)


def ptrs(v):
    return None if v is None else (C.c_void_p * max(1, len(v)))(*v)


def test_record_layout():
    for l in (LAY, p8.Layout(1, 1, 32, 1), p8.Layout(3, 2, 128, 32), p8.Layout(1, 16, 128, 769)):
        rows = -(-l.capacity // 32) * 32
        heads = l.kv_layers * 2 * l.n_kv_heads
        want = heads * rows * l.head_dim + heads * rows // 32 * 4 + rows // 32 * 4
        assert l.record_bytes == -(-want // 128) * 128 and l.rows == rows
        pool = torch.zeros((3, l.record_bytes), dtype=torch.uint8)
        codes, scales, words = p8.views(l, pool)
        assert codes.shape == (3, l.kv_layers, 2, l.n_kv_heads, rows, l.head_dim) and codes.dtype == torch.uint8
        assert scales.shape == (3, l.kv_layers, 2, l.n_kv_heads, rows // 32) and words.shape == (3, rows // 32)
        codes[2, -1, 1, -1, -1, -1] = 7
        scales[2, 0, 0, 0, 0] = 1.5
        words[2, -1] = 9
        at = pool[2].numpy()
        assert at[heads * rows * l.head_dim - 1] == 7
        assert at[heads * rows * l.head_dim:][:4].view(np.float32)[0] == 1.5
        assert at[heads * rows * l.head_dim + heads * rows // 32 * 4:][:rows // 8].view(np.int32)[-1] == 9


@pytest.mark.parametrize("kw", [dict(kv_layers=0), dict(n_kv_heads=0), dict(head_dim=48), dict(head_dim=256), dict(capacity=0),
                                dict(capacity=(1 << 24) + 1), dict(kv_layers=5000), dict(n_kv_heads=5000), dict(capacity=-5)])
def test_layouts_that_are_refused(kw):
    assert L.ebrl_prefix8_record_bytes(lay(**kw)) == 0
    assert len(L.ebrl_prefix8_last_error()) > 0
    with pytest.raises(B.EbrlError):
        p8.new_pool(LAY._replace(**kw), 2, device="cpu")


def quantize(**kw):
    a = dict(lay=lay(), pool=P0, n_slots=4, n=3, slots=None, planes=[P0] * 3, len=[1, 100, 0], rows=None, rs=0, dt=B.BF16, mask=None, quota=0)
    a.update(kw)
    return L.ebrl_prefix8_quantize(a["lay"], a["pool"], a["n_slots"], a["n"], ints(a["slots"]), ptrs(a["planes"]), ints(a["len"]), ints(a["rows"]), a["rs"],
                                   a["dt"], ptrs(a["mask"]), a["quota"], None)


def attend(**kw):
    a = dict(lay=lay(), pool=P0, n_slots=4, n=3, slots=None, len=[1, 100, 0], layer=1, q=P0, dt=B.BF16, H=8, heads=8, qe=4096, qt=512, out=P0 + 65536,
             oe=4096, ot=512, lse=P0, scale=0.125, split=-1, ws=None, wsb=0, quota=0)
    a.update(kw)
    return L.ebrl_prefix8_attend(a["lay"], a["pool"], a["n_slots"], a["n"], ints(a["slots"]), ints(a["len"]), a["layer"], a["q"], a["dt"], a["H"], a["heads"],
                                 a["qe"], a["qt"], a["out"], a["oe"], a["ot"], a["lse"], a["scale"], a["split"], a["ws"], a["wsb"], a["quota"], None)


def weigh(**kw):
    a = dict(lay=lay(), pool=P0, n_slots=4, n=3, slots=None, len=[1, 100, 0], layer=0, q=P0, dt=B.F32, H=8, heads=8, qe=4096, qt=512, lse=P0, le=64, lt=8, lh=1,
             scale=0.125, w=P0, ws=100, acc=1, quota=0)
    a.update(kw)
    return L.ebrl_prefix8_weigh(a["lay"], a["pool"], a["n_slots"], a["n"], ints(a["slots"]), ints(a["len"]), a["layer"], a["q"], a["dt"], a["H"], a["heads"],
                                a["qe"], a["qt"], a["lse"], a["le"], a["lt"], a["lh"], a["scale"], a["w"], a["ws"], a["acc"], a["quota"], None)


def evict(**kw):
    a = dict(lay=lay(), src=P0, dst=1 << 40, n_slots=4, n=3, slots=None, len=[1, 100, 0], keep=[1, 50, 7], pf=0, pl=0, w=P0, ws=100, wo=None, wos=0, kept=P0,
             ks=50, quota=0)
    a.update(kw)
    return L.ebrl_prefix8_evict(a["lay"], a["src"], a["dst"], a["n_slots"], a["n"], ints(a["slots"]), ints(a["len"]), ints(a["keep"]), a["pf"], a["pl"], a["w"],
                                a["ws"], a["wo"], a["wos"], a["kept"], a["ks"], a["quota"], None)


CALLS = {"quantize": quantize, "attend": attend, "weigh": weigh, "evict": evict}
COMMON = [dict(lay=None), dict(n=-1), dict(n_slots=-1), dict(n_slots=2), dict(len=None), dict(len=[1, 101, 0]), dict(len=[1, -1, 0]), dict(slots=[0, 4, 1]),
          dict(slots=[0, -1, 1])]
REFUSED = {
    "quantize": [dict(pool=None), dict(pool=P0 + 8), dict(slots=[1, 2, 1]), dict(planes=None), dict(planes=[P0, None, P0]), dict(planes=[P0, P0 + 8, P0]), dict(dt=2), dict(rs=255),
                 dict(rs=260), dict(rs=-256), dict(rows=[1, 99, 0])],
    "attend": [dict(pool=None), dict(layer=2), dict(layer=-1), dict(q=None), dict(q=P0 + 2), dict(dt=2), dict(H=0), dict(heads=6), dict(heads=0), dict(qe=4095), dict(qt=-512),
               dict(out=None), dict(out=P0 + 4), dict(oe=4092), dict(ot=256), dict(oe=512, ot=512), dict(lse=P0 + 2), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(split=-2), dict(split=100), dict(out=P0, oe=8192)],
    "weigh": [dict(slots=[1, 2, 1]), dict(layer=2), dict(q=None), dict(lse=None), dict(lse=P0 + 1), dict(w=None), dict(w=P0 + 2), dict(ws=99), dict(le=-1), dict(lt=-1), dict(lh=-1),
              dict(scale=float("nan")), dict(qt=510)],
    "evict": [dict(src=None), dict(dst=None), dict(dst=P0 + 128), dict(slots=[1, 2, 1]), dict(keep=None), dict(keep=[1, -1, 0]), dict(pf=-1), dict(pl=-1), dict(w=None), dict(kept=None),
              dict(ws=99), dict(wo=1 << 30, wos=99), dict(wo=P0, wos=200), dict(wo=P0 + 4, wos=100), dict(ks=49), dict(kept=P0 + 2)],
}


@pytest.mark.parametrize("op", list(CALLS))
def test_invalid_arguments_are_refused_before_the_device(op):
    for kw in COMMON + REFUSED[op]:
        st = CALLS[op](**kw)
        assert st == B.ERR_INVALID_ARG, (op, kw, st)
        assert len(L.ebrl_prefix8_last_error()) > 0
    assert CALLS[op](quota=-1) == B.ERR_QUOTA
    assert CALLS[op](lay=lay(head_dim=96)) == B.ERR_UNSUPPORTED
    assert CALLS[op](n=0) == B.OK                      # nothing to do, whatever else is given
    assert CALLS[op](n=0, len=None, slots=None) == B.OK
    if op in ("attend", "weigh"):
        assert CALLS[op](H=1025, heads=4) == B.ERR_UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="this check is for a box without a GPU")
def test_valid_calls_fail_loudly_without_a_device():
    for op in CALLS:
        assert CALLS[op]() == B.ERR_CUDA, op
    assert attend(slots=[1, 1, 1]) == B.ERR_CUDA       # readers may share a slot
    assert attend(out=P0) == B.ERR_CUDA                # in place
    assert attend(oe=512, ot=2048) == B.ERR_CUDA       # token-major outputs
    assert evict(dst=P0) == B.ERR_CUDA                 # in place
    assert evict(wo=P0, wos=100) == B.ERR_CUDA


def test_binding_refusals():
    pool = torch.zeros((2, LAY.record_bytes), dtype=torch.uint8)
    for bad in (pool, pool[:, :-1], pool.float()):     # host memory; not records; not bytes
        with pytest.raises(ValueError):
            p8.attend(LAY, bad, torch.zeros((1, 1, 4, 64)), [1])
    with pytest.raises(B.EbrlError):
        p8.quantize(LAY._replace(head_dim=40), pool, torch.zeros((1, 2, 2, 3, 160)))
    assert p8._host([1, 2], "x").dtype == torch.int32
    for bad in (torch.zeros(2), torch.zeros((1, 2), dtype=torch.int32), [2 ** 40]):
        with pytest.raises((ValueError, OverflowError)):
            p8._host(bad, "x")


def test_handle_configuration_rules():
    def cfg(**kw):
        base = dict(H=8, A=7, d=256, n_layers=2, n_heads=4, K_steps=4, max_prefix_len=64, max_group_envs=16, kv_dtype=B.E4M3)
        base.update(kw)
        return B.make_cfg(**base)
    check = lambda c: B.lib().ebrl_actgen_check_cfg(C.byref(c))   # noqa: E731
    assert check(cfg()) == B.OK and check(cfg(dtype=B.BF16)) == B.OK and check(cfg(kv_layers=2)) == B.OK
    assert check(cfg(d_ctx=128)) == B.ERR_UNSUPPORTED
    assert check(cfg(kv_dtype=3)) == B.ERR_INVALID_ARG
    assert check(cfg(dtype=B.BF16, kv_dtype=B.F32)) == B.ERR_UNSUPPORTED
    assert check(cfg(max_prefix_len=(1 << 24) + 1)) == B.ERR_UNSUPPORTED
    bad = cfg()
    bad.param_dtype = B.E4M3
    assert check(bad) == B.ERR_INVALID_ARG
    assert p8.layout_for(cfg(kv_layers=2)) == p8.Layout(2, 4, 64, 64)
    assert B.lib().ebrl_actgen_submit_weighed(None, 0, None, None, None, None, None, 0, None, None) == B.ERR_INVALID_ARG


def test_the_reference_itself():
    """e4m3 against torch's, the scale rule at its border, and selection with ties."""
    x = torch.cat([torch.randn(20000) * 100, torch.linspace(-500, 500, 4001), torch.tensor([0.0, -0.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, 448.0, 464.0, float("nan")])])
    want = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = ref.encode(x.double().numpy())
    assert ((got == want) | ((got & 127 == 127) & (want & 127 == 127))).all()
    assert ref.block_scale(448.0) == 1.0 and ref.block_scale(448.0001) == 2.0 and ref.block_scale(224.0) == 0.5 and ref.block_scale(0.0) == 1.0
    assert ref.block_scale(1e-45) == 2.0 ** -126
    assert ref.select([1, 3, 3, 0, float("nan")], [1, 1, 1, 1, 1], 5, 2, 0, 0) == [1, 2]
    assert ref.select([1, 3, 3, 0, 9], [1, 0, 1, 1, 0], 5, 3, 0, 1) == [0, 2, 4]
