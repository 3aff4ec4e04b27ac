"""GPU tests of handles on 8-bit prefix records: cross-attention through a whole action head against the fp64 oracle on the
records' values, and the token weights that a submit adds up."""
import math

import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import TOL
from helpers import chunk_rel_err, np32, oracle_cfg, oracle_weights
from paper_2609_27547_b200 import binding as B
from paper_2609_27547_b200 import prefix8 as p8
from paper_2609_27547_b200 import synth

pytestmark = pytest.mark.gpu


def values_of(lay, pool, i, P):
    """The planes [kv_layers, 2, P, d] that record i stands for, fp32 (exact: four significant bits times a power of two)."""
    codes, scales, _ = p8.views(lay, pool.cpu())
    x = codes[i, ..., :P, :].contiguous().view(torch.float8_e4m3fn).float() * scales[i].abs().repeat_interleave(32, -1)[..., :P, None]
    return x.transpose(2, 3).reshape(lay.kv_layers, 2, P, -1)


class Case:
    def __init__(self, dtype="bf16", B_=12, H=8, d=256, heads=4, L=2, K=3, P=(1, 90), kv_layers=1, flags=0, hide=0.0, inflight=2, mixed=True, cap=None):
        self.w = synth.scaled(synth.WORKLOADS[0], B=B_, dtype=dtype, H=H, d=d, n_heads=heads, L=L, K=K, P=P, mixed_steps=mixed)
        self.wt = synth.make_weights(self.w, random_gains=True)
        self.envs = [synth.make_env(self.w, e) for e in range(B_)]
        self.cfg = B.cfg_for(self.w, max_group_envs=B_, max_inflight_groups=inflight, flags=flags, kv_dtype=B.E4M3)
        self.cfg.kv_layers = kv_layers
        self.cfg.max_prefix_len = cap or max(e.P for e in self.envs)
        self.kv_layers = kv_layers
        self.lay = p8.layout_for(self.cfg)
        g = torch.Generator().manual_seed(3)
        planes = [e.kv.view(1, 2, e.P, d).expand(kv_layers, 2, e.P, d) if kv_layers == 1 else torch.randn((kv_layers, 2, e.P, d), generator=g).to(e.kv.dtype) for e in self.envs]
        self.P = [e.P for e in self.envs]
        self.mask = [(torch.rand(p, generator=g) >= hide).to(torch.uint8) for p in self.P]
        for m in self.mask:
            m[0] = 1
        self.pool = p8.new_pool(self.lay, B_)
        self.pool.fill_(0x7f)
        p8.quantize(self.lay, self.pool, [x.cuda().contiguous() for x in planes], self.P, mask=[m.cuda() for m in self.mask])
        self.noise = torch.stack([e.noise for e in self.envs]).cuda()
        self.steps = [e.step for e in self.envs]

    def seen(self, i):
        return self.mask[i][:self.P[i]].bool()

    def reference(self, ids, kv=None):
        oc = oracle_cfg(self.w)
        oc.kv_layers = self.kv_layers
        kv = kv or [values_of(self.lay, self.pool, i, self.P[i])[:, :, self.seen(i)] for i in ids]
        return oracle.actgen(oc, oracle_weights(self.wt), [np32(x) for x in kv], np.stack([np32(self.envs[i].noise) for i in ids]),
                             step_index=[self.steps[i] for i in ids])

    def run(self, gen, groups, quota=0, weights=None, stream=None):
        out = torch.full_like(self.noise, 9.0)
        for g in groups:
            o = torch.empty((len(g),) + tuple(self.noise.shape[1:]), device="cuda")
            gen.submit(g, [self.pool[i] for i in g], self.noise[g].contiguous(), o, sm_quota=quota, prefix_len=[self.P[i] for i in g],
                       step_index=[self.steps[i] for i in g], prefix_weight=None if weights is None else [weights[i] for i in g], stream=stream)
            gen.sync()
            out[g] = o
        return out.cpu().numpy()


@pytest.mark.parametrize("kw", [
    dict(dtype="bf16", H=8, d=256, heads=4),
    dict(dtype="bf16", H=16, d=256, heads=2, kv_layers=2),
    dict(dtype="bf16", H=20, d=256, heads=8, hide=0.4),
    dict(dtype="bf16", H=1, d=128, heads=2, flags=B.FLAG_FORCE_SIMT),
    dict(dtype="f32", H=8, d=256, heads=4, hide=0.4),
    dict(dtype="f32", H=16, d=256, heads=2, kv_layers=2),
    dict(dtype="f32", H=32, d=128, heads=4, flags=B.FLAG_FORCE_SIMT),
    dict(dtype="f32", H=3, d=128, heads=4, K=1, P=(1, 3)),
    dict(dtype="bf16", H=8, d=256, heads=4, flags=B.FLAG_DEBUG_CANARY, P=(100, 400), cap=500),
])
def test_handle_against_the_oracle(kw):
    c = Case(**kw)
    gen = B.ActGen(c.cfg, c.wt)
    got = c.run(gen, [list(range(12))])
    gen.destroy()
    assert chunk_rel_err(got, c.reference(range(12))) <= TOL[kw["dtype"]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_handle_results_do_not_depend_on_groups_quota_or_weights(dtype):
    c = Case(dtype=dtype, P=(1, 200))
    gen = B.ActGen(c.cfg, c.wt)
    base_w = torch.zeros((12, c.cfg.max_prefix_len), device="cuda")
    base = c.run(gen, [list(range(12))], weights=base_w)
    assert np.array_equal(c.run(gen, [list(range(12))]), base)
    for quota, groups in ((16, [[3, 1, 2], [0, 11, 10, 9], [4, 5, 6, 7, 8]]), (74, [[i] for i in range(11, -1, -1)]), (148, [list(range(11, -1, -1))])):
        w = torch.zeros_like(base_w)
        assert np.array_equal(c.run(gen, groups, quota=quota, weights=w), base)
        assert torch.equal(w, base_w)
    gen.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_weights_of_a_submit(dtype):
    """Every row's weights sum to 1: an environment's weights sum to rows x heads x layers x steps, all on visible tokens; they are added to
    what is there; environments without an array are left out.  With W_qc = 0 the weights are uniform."""
    c = Case(dtype=dtype, hide=0.3, K=3, L=2, P=(5, 90))
    cap = c.cfg.max_prefix_len
    gen = B.ActGen(c.cfg, c.wt)
    w = torch.full((12, cap + 1), 2.0, device="cuda")
    arrays = [w[i, :cap] if i % 3 else None for i in range(12)]
    c.run(gen, [list(range(12))], weights=arrays)
    for i in range(12):
        steps = 3 - c.steps[i]
        vis = torch.zeros(cap + 1, dtype=torch.bool)
        vis[:c.P[i]] = c.seen(i)
        added = w[i].cpu() - 2.0
        if i % 3 == 0:
            assert (added == 0).all()
            continue
        assert (added[~vis] == 0).all() and (added[vis] > 0).all()
        want = c.w.H * c.w.n_heads * c.w.L * steps
        assert abs(float(added.double().sum()) - want) <= 1e-4 * want
    gen.destroy()
    for l in c.wt["layers"]:
        l["w_qc"].zero_()
    gen = B.ActGen(c.cfg, c.wt)
    w = torch.zeros((12, cap), device="cuda")
    c.run(gen, [list(range(12))], weights=w)
    for i in range(12):
        n = int(c.seen(i).sum())
        want = c.w.H * c.w.n_heads * c.w.L * (3 - c.steps[i]) / n
        assert torch.allclose(w[i, :c.P[i]].cpu()[c.seen(i)], torch.tensor(want), rtol=1e-5, atol=0)
    gen.destroy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_generate_shorten_generate(dtype):
    """Records are halved by the weights of one generation, and the next one runs on what is left."""
    c = Case(dtype=dtype, P=(40, 120), mixed=False)
    gen = B.ActGen(c.cfg, c.wt)
    w = torch.zeros((12, c.cfg.max_prefix_len), device="cuda")
    c.run(gen, [list(range(12))], weights=w)
    before = w.clone()
    new, kept = p8.evict(c.lay, c.pool, c.pool, w, c.P, [p // 2 for p in c.P], weight_out=w)
    for i in range(12):
        k = kept[i, :int(new[i])].long()
        top = before[i, :c.P[i]].topk(int(new[i])).values.min()
        assert (before[i, k] >= top).all() and (k[1:] > k[:-1]).all() and torch.equal(w[i, :int(new[i])], before[i, k])
    c.P = new.tolist()
    c.mask = [torch.ones(p, dtype=torch.uint8) for p in c.P]
    got = c.run(gen, [list(range(12))])
    gen.destroy()
    assert chunk_rel_err(got, c.reference(range(12))) <= TOL[dtype]


def test_host_records_queue_and_scattered_submits():
    c = Case(dtype="bf16", mixed=False)
    gen = B.ActGen(c.cfg, c.wt)
    base = c.run(gen, [list(range(12))])
    host = c.pool.cpu().pin_memory()
    out = torch.empty_like(c.noise.cpu()).pin_memory()
    gen.submit_host(list(range(12)), [host[i] for i in range(12)], c.noise.cpu().pin_memory(), out, prefix_len=c.P, step_index=c.steps)
    gen.sync()
    assert np.array_equal(out.numpy(), base)
    q = B.Queue(gen, capacity=16, max_group=5)
    res = torch.empty_like(c.noise)
    t = [q.push(i, c.pool[i], c.P[i], c.noise[i], res[i], c.steps[i]) for i in range(12)]
    for x in t:
        assert q.wait(x, 20000) == B.OK
    q.destroy()
    torch.cuda.synchronize()
    assert np.array_equal(res.cpu().numpy(), base)
    gen.destroy()


def test_submit_refusals_on_a_device():
    c = Case(dtype="bf16", B_=12, mixed=False, inflight=4)
    gen = B.ActGen(c.cfg, c.wt)
    o = torch.empty_like(c.noise)
    w = torch.zeros((12, c.cfg.max_prefix_len), device="cuda")
    with pytest.raises(ValueError):
        gen.submit([0], [c.pool[0]], c.noise[:1], o[:1])                                     # no length
    with pytest.raises(ValueError):
        gen.submit([0], [c.pool[0, :-128]], c.noise[:1], o[:1], prefix_len=[c.P[0]])         # not a record
    with pytest.raises(B.EbrlError) as e:                                                    # one array for two environments
        gen.submit([0, 1], [c.pool[0], c.pool[1]], c.noise[:2], o[:2], prefix_len=c.P[:2], prefix_weight=[w[0], w[0]])
    assert e.value.status == B.ERR_INVALID_ARG
    gen.submit([0], [c.pool[0]], c.noise[:1], o[:1], prefix_len=c.P[:1], prefix_weight=[w[0]])
    with pytest.raises(B.EbrlError):                                                         # ... or for one queued already
        gen.submit([1], [c.pool[1]], c.noise[1:2], o[1:2], prefix_len=c.P[1:2], prefix_weight=[w[0]])
    gen.sync()
    gen.destroy()
    plain = B.ActGen(B.cfg_for(c.w, max_group_envs=12), c.wt)
    with pytest.raises(B.EbrlError) as e:
        plain.submit([0], [c.envs[0].kv.cuda().contiguous()], c.noise[:1], o[:1], prefix_weight=[torch.zeros(4096, device="cuda")])
    assert e.value.status == B.ERR_UNSUPPORTED
    plain.destroy()
