"""CPU-only tests of the 8-bit prefix operators: calls that have to be let through (arguments are checked before anything touches a
device, so without one a valid call ends with a CUDA error), and what the binding hands to the library."""
import gc
import weakref

import pytest
import torch

from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import prefix8 as p8
from test_prefix8_host import LAY, P0, attend, evict, weigh
from test_queue_host import FakeBackend

no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="this check is for a box without a GPU")


class Pool:
    """What the binding asks of a pool."""
    device = torch.device("cuda", 0)
    dtype = torch.uint8
    shape = (2, LAY.record_bytes)

    def dim(self):
        return 2

    def is_contiguous(self):
        return True


def test_a_layout_in_use_outlives_the_cache():
    """Other threads may use any number of layouts between a call's check of its pool and the call itself."""
    held = p8._pool(LAY, Pool())
    alive = weakref.ref(p8._record(LAY)[0])
    for i in range(600):
        p8._record(LAY._replace(capacity=1000 + i))
    gc.collect()
    assert alive() is not None
    del held
    gc.collect()
    assert alive() is None


@no_device
def test_strides_of_a_single_environment_or_token_do_not_matter():
    for call in (attend, weigh):
        assert call(n=1, len=[7], qe=3) == B.ERR_CUDA
        assert call(n=1, len=[7], qe=-8) == B.ERR_CUDA
        assert call(H=1, qt=3) == B.ERR_CUDA
        assert call(n=1, len=[7], H=1, qe=1, qt=1) == B.ERR_CUDA
        assert call(qe=4095) == B.ERR_INVALID_ARG and call(qt=511) == B.ERR_INVALID_ARG
        assert call(n=1, len=[7], qt=511) == B.ERR_INVALID_ARG and call(H=1, qe=4095) == B.ERR_INVALID_ARG
    assert attend(n=1, len=[7], oe=3) == B.ERR_CUDA and attend(H=1, ot=3) == B.ERR_CUDA
    assert attend(n=1, len=[7], ot=511) == B.ERR_INVALID_ARG and attend(H=1, oe=4095) == B.ERR_INVALID_ARG


@no_device
def test_weigh_without_query_rows():
    assert weigh(H=0, acc=0) == B.ERR_CUDA
    assert weigh(H=0, acc=0, q=None, lse=None) == B.ERR_CUDA
    assert weigh(H=3, heads=0, acc=0, q=None, lse=None) == B.ERR_CUDA
    for kw in (dict(slots=[1, 2, 1]), dict(w=None), dict(ws=99), dict(layer=2), dict(len=[1, 101, 0]), dict(dt=2), dict(H=-1), dict(heads=-4)):
        assert weigh(**{**dict(H=0, acc=0), **kw}) == B.ERR_INVALID_ARG, kw
    assert attend(H=0) == B.ERR_INVALID_ARG and attend(heads=0) == B.ERR_INVALID_ARG


@no_device
def test_evict_weights_next_to_one_another():
    assert evict(ws=200, wo=P0 + 400, wos=200) == B.ERR_CUDA          # [n_slots][2][capacity], either way round
    assert evict(w=P0 + 400, ws=200, wo=P0, wos=200) == B.ERR_CUDA
    assert evict(ws=250, wo=P0 + 500, wos=250) == B.ERR_CUDA
    assert evict(ws=200, wo=P0 + 4 * 700, wos=100) == B.ERR_CUDA      # right behind the last row's capacity
    for kw in (dict(ws=200, wo=P0 + 396, wos=200), dict(ws=200, wo=P0 + 404, wos=200), dict(ws=150, wo=P0 + 400, wos=150), dict(ws=200, wo=P0 + 400, wos=100),
               dict(ws=200, wo=P0 + 4 * 699, wos=100), dict(wo=P0 + 4, wos=100), dict(w=P0 + 4, wo=P0, wos=100)):
        assert evict(**kw) == B.ERR_INVALID_ARG, kw


def test_a_queue_takes_records_of_its_handle_only():
    """What a queue's handle reads is a whole record, whatever the prefix's length: planes, a record of another layout or a part of one are refused
    like in a submit (raw addresses are the caller's word)."""
    gen = object.__new__(B.ActGen)
    gen._h, gen._record_bytes = None, None
    gen.cfg = B.make_cfg(H=8, A=7, d=256, n_layers=2, n_heads=4, K_steps=4, max_prefix_len=64, max_group_envs=16, kv_dtype=B.E4M3)
    size = p8.layout_for(gen.cfg).record_bytes
    be = FakeBackend()
    q = B.Queue(gen, capacity=8, max_group=4, backend=be.struct)
    pool, state = torch.zeros((2, size), dtype=torch.uint8), torch.zeros((2, 8, 7))
    for bad in (torch.zeros((1, 2, 5, 256)), pool[0, :-128], torch.zeros(size * 2, dtype=torch.uint8)[::2], pool):
        for push in (q.push, q.try_push):
            with pytest.raises(ValueError):
                push(1, bad, 5, state[0], state[1], 0)
    assert q.wait(q.push(1, pool[0], 5, state[0], state[1], 0)) == B.OK
    assert q.wait(q.push(2, pool[1].data_ptr(), 5, state[0], state[1], 0)) == B.OK
    assert q.wait(q.try_push(3, pool[1], 5, state[0], state[1], 0)[1]) == B.OK
    q.destroy()
    assert [e for g in be.groups for e in g["ids"]] == [1, 2, 3]
