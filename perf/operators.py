"""What the operators on 8-bit prefix caches are measured on.

A prefix cache holds, per environment, one record: e4m3 codes [kv_layers][2][kv_heads][rows][head_dim] (keys, then
values; rows = the capacity rounded up to 32), an fp32 scale for each block of 32 tokens and head, and one bit per token
that says whether queries may see it.  A pool is a uint8 tensor [n_slots, record_bytes].  Four operators work on it:

  quantize  planes [kv_layers][2][P][kv_heads * head_dim] -> record
  attend    softmax(scale q k^T) v over the record's visible tokens, and the log-sum-exp of each row
  weigh     the weight every token got from those queries, summed over rows and heads
  evict     keep the tokens of the largest weight, in their order, in a shorter record
"""
import math

import torch

own = False

BLOCK = 32
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the record, and the cases --------------------------------------------------------------------------------------

def sizes(c):
    rows = -(-c["cap"] // BLOCK) * BLOCK
    codes = c["layers"] * 2 * c["kvh"] * rows * c["hd"]
    scales = c["layers"] * 2 * c["kvh"] * (rows // BLOCK) * 4
    mask = rows // BLOCK * 4
    return rows, codes, scales, mask, -(-(codes + scales + mask) // 128) * 128


def views(c, pool):
    """(codes as uint8, scales, mask words) of a pool."""
    rows, nc, ns, nm, _ = sizes(c)
    n, nb = pool.shape[0], rows // BLOCK
    return (pool[:, :nc].unflatten(1, (c["layers"], 2, c["kvh"], rows, c["hd"])),
            pool[:, nc:nc + ns].view(torch.float32).unflatten(1, (c["layers"], 2, c["kvh"], nb)),
            pool[:, nc + ns:nc + ns + nm].view(torch.int32))


def lengths(c, seed):
    """The prefix lengths (host): all the longest, or spread from `lo` to it."""
    g = torch.Generator().manual_seed(seed * 2 + 1)
    lens = torch.randint(c["lo"], c["len"] + 1, (c["n"],), generator=g, dtype=torch.int32)
    lens[-1] = c["len"]
    return lens


def listed():
    def case(name, op, n, lo, length, kvh, hd, layers=1, cap=0, **kw):
        return dict(name=name, op=op, n=n, lo=lo, len=length, cap=cap or length, kvh=kvh, hd=hd, layers=layers, **kw)
    return [
        # one environment was reset: its short observation is written, from an fp32 backbone
        case("quantize_one_f32", "quantize", 1, 37, 37, 4, 64, layers=2, cap=64, dtype="f32", hide=0.0),
        # the observations of a group of the large bf16 head, with padded camera tokens hidden
        case("quantize_group_bf16", "quantize", 128, 700, 768, 16, 128, dtype="bf16", hide=0.1),
        # one robot asks for one action token: latency
        case("attend_one_token", "attend", 1, 256, 256, 16, 64, dtype="bf16", H=1, G=1, hide=0.0),
        # the mid-size bf16 head, a batch of environments with 8 action tokens each
        case("attend_mid_bf16", "attend", 256, 256, 256, 16, 64, dtype="bf16", H=8, G=1, hide=0.0),
        # the small fp32 head on ragged prefixes
        case("attend_ragged_f32", "attend", 512, 64, 512, 4, 64, dtype="f32", H=8, G=1, hide=0.0),
        # the large bf16 head: a queue of groups with 16 action tokens each
        case("attend_large_bf16", "attend", 512, 768, 768, 16, 128, dtype="bf16", H=16, G=1, hide=0.0),
        # two long histories, one token, four query heads on each key/value head
        case("attend_long_shared_heads", "attend", 2, 60001, 65537, 4, 128, dtype="bf16", H=1, G=4, hide=0.0),
        # padded observations: most tokens hidden, some environments see nothing at all
        case("attend_padded", "attend", 96, 0, 301, 2, 32, dtype="bf16", H=32, G=2, hide=0.7),
        # the weights that the prefix tokens of a few small fp32 environments got
        case("weigh_few_f32", "weigh", 16, 20, 32, 4, 64, dtype="f32", H=8, G=1, hide=0.0, add=False),
        # the same for a group of the large bf16 head, added to what earlier steps gave
        case("weigh_group_bf16", "weigh", 256, 700, 768, 16, 128, dtype="bf16", H=16, G=1, hide=0.1, add=True),
        # one environment's cache is cut to its heaviest 100 tokens
        case("evict_one", "evict", 1, 256, 256, 16, 64, keep=100, first=4, last=8, hide=0.0),
        # a group's caches are halved
        case("evict_group", "evict", 128, 700, 768, 16, 128, keep=384, first=0, last=16, hide=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "attend", "attend", "attend", "weigh", "evict"])
    hd = rng.choice([32, 64, 128])
    kvh = rng.choice([1, 2, 4, 8, 16])
    layers = rng.choice([1, 1, 2])
    length = _log(rng, 1, 2000) if rng.random() < 0.8 else _log(rng, 2000, 70000)
    room = 400e6 if op == "attend" else 120e6
    most = max(1, int(room / (2 * layers * kvh * hd * length)))
    n = _log(rng, 1, min(most, 600))
    c = dict(op=op, n=n, lo=rng.choice([0, length // 2, length]), len=length, cap=length + rng.choice([0, 0, 1, 40]), kvh=kvh, hd=hd,
             layers=layers, hide=rng.choice([0.0, 0.0, 0.1, 0.6]))
    if op != "evict":
        c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
    if op in ("attend", "weigh"):
        c["H"] = rng.choice([1, 1, 2, 7, 8, 16, 19, 32])
        c["G"] = rng.choice([1, 1, 2, 4])
        while n * c["H"] * c["G"] * kvh * length > 1.2e8:   # the plain form's scores
            c["H"], c["G"] = max(1, c["H"] // 2), max(1, c["G"] // 2)
            if c["H"] * c["G"] == 1:
                break
    if op == "weigh":
        c["add"] = rng.random() < 0.5
    if op == "evict":
        c["keep"] = rng.randint(0, length + 3)
        c["first"], c["last"] = rng.choice([(0, 0), (1, 0), (4, 16)])
    return c


def work(c):
    # ragged lengths are uniform between lo and len
    tokens = c["n"] * (c["lo"] + c["len"]) / 2
    d = c["kvh"] * c["hd"]
    if c["op"] == "quantize":
        per = 2 * c["layers"] * d
        return {"bytes": tokens * per * ((4 if c["dtype"] == "f32" else 2) + 1 + 4 / (BLOCK * c["hd"])), "flops": tokens * per * 2}
    if c["op"] == "evict":
        kept = min(c["keep"], (c["lo"] + c["len"]) / 2) * c["n"]
        return {"bytes": 2 * kept * 2 * c["layers"] * d * (1 + 4 / (BLOCK * c["hd"])) + 4 * tokens + 8 * kept, "flops": kept * 2 * c["layers"] * d}
    esz = 4 if c["dtype"] == "f32" else 2
    rows = c["n"] * c["H"] * c["G"] * c["kvh"]
    if c["op"] == "attend":
        return {"bytes": 2 * tokens * d * (1 + 4 / (BLOCK * c["hd"])) + rows * (2 * c["hd"] * esz + 4), "flops": 4.0 * c["H"] * c["G"] * tokens * d}
    return {"bytes": tokens * d * (1 + 4 / (BLOCK * c["hd"])) + rows * (c["hd"] * esz + 4) + tokens * 4 * (2 if c["add"] else 1),
            "flops": 2.0 * c["H"] * c["G"] * tokens * d}


# ---- plain forms -------------------------------------------------------------------------------------------------------

def block_scale(amax):
    """The power of two s with amax / s in (224, 448]; 1 where amax is 0."""
    m, e = torch.frexp(amax)   # amax = m 2^e, m in [0.5, 1)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp_min(-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.ones_like(amax))


def codes_of(x, s):
    """e4m3 of x / s, saturated (s is a power of two, the quotient is exact)."""
    return (x / s).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def seen(c, lens, words):
    """[n, rows]: which tokens queries see."""
    t = torch.arange(sizes(c)[0], device=words.device)
    bits = (words[:, t // BLOCK] >> (t % BLOCK).to(torch.int32)) & 1
    return (bits == 1) & (t < lens.to(words.device)[:, None])


def pack_bits(m):
    """[n, rows] truth values -> [n, rows / 32] words."""
    w = m.unflatten(1, (-1, BLOCK)).to(torch.int64) << torch.arange(BLOCK, device=m.device)
    w = w.sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def plain_quantize(c, pool, x, lens, visible):
    """x [n, layers, 2, rows, kvh * hd] in 32 bits, rows past the lengths whatever; visible [n, rows]."""
    codes, scales, words = views(c, pool)
    n, rows = x.shape[0], x.shape[3]
    t = torch.arange(rows, device=x.device)
    inside = t < lens.to(x.device)[:, None]
    use = (visible & inside)[:, None, None, :, None]
    x = torch.where(use, x, torch.zeros((), device=x.device)).unflatten(-1, (c["kvh"], c["hd"])).transpose(3, 4)   # [n, layers, 2, kvh, rows, hd]
    a = x.abs()
    a = torch.where(torch.isfinite(a), a, torch.zeros((), device=x.device)).unflatten(4, (-1, BLOCK)).amax((-1, -2))
    s = block_scale(a)
    q = codes_of(x, s.repeat_interleave(BLOCK, 4)[..., None])
    codes.copy_(torch.where(inside[:, None, None, None, :, None], q, codes))
    live = inside[:, ::BLOCK]
    scales.copy_(torch.where(live[:, None, None, None, :], s, scales))
    words.copy_(torch.where(live, pack_bits(visible & inside), words))


def scores(c, state):
    """(scale q k^T with hidden tokens at -inf, the values) of the case's layer, in 32 bits."""
    codes, sc, words = views(c, state["pool"])
    kv = codes[:, state["layer"]].view(torch.float8_e4m3fn).float() * sc[:, state["layer"]].repeat_interleave(BLOCK, -1)[..., None]
    ok = seen(c, state["lens"], words)
    kv = torch.where(ok[:, None, None, :, None], kv, torch.zeros((), device=kv.device))
    n, H = state["q"].shape[:2]
    q = state["q"].float().view(n, H, c["kvh"], c["G"], c["hd"]).permute(0, 2, 1, 3, 4).reshape(n, c["kvh"], H * c["G"], c["hd"])
    s = q @ kv[:, 0].transpose(-1, -2) * (1.0 / math.sqrt(c["hd"]))
    return torch.where(ok[:, None, None, :], s, torch.full((), -math.inf, device=s.device)), kv[:, 1]


def per_row(c, x, H):
    """[n, kvh, H * G, ...] -> [n, H, heads, ...]"""
    return x.unflatten(2, (H, c["G"])).transpose(1, 2).flatten(2, 3)


def plain_attend(c, state):
    s, v = scores(c, state)
    m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    p = torch.exp(s - m)
    z = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(z > 0, z, torch.ones_like(z))
    H = state["q"].shape[1]
    return per_row(c, o, H).to(state["q"].dtype), per_row(c, (m + torch.log(z)).squeeze(-1), H)


def plain_weigh(c, state):
    s, _ = scores(c, state)
    n, H = state["q"].shape[:2]
    lse = state["lse"].view(n, H, c["kvh"], c["G"]).permute(0, 2, 1, 3).flatten(2, 3)[..., None]
    p = torch.where(s > -math.inf, torch.exp(s - lse), torch.zeros((), device=s.device))
    w = p.sum((1, 2))[:, :c["cap"]]
    inside = torch.arange(c["cap"], device=s.device) < state["lens"].to(s.device)[:, None]
    state["weight"].copy_(torch.where(inside, w + (state["weight"] if c["add"] else 0), state["weight"]))
    return state["weight"]


def plain_evict(c, state):
    codes, sc, words = views(c, state["pool"])
    to_codes, to_sc, to_words = views(c, state["dst"])
    dev, cap, rows = codes.device, c["cap"], codes.shape[4]
    lens, new = state["lens"].to(dev)[:, None], torch.minimum(state["lens"], state["keep"]).to(dev)[:, None]
    t = torch.arange(cap, device=dev)
    low = torch.full((), -math.inf, device=dev)
    ok = seen(c, state["lens"], words)[:, :cap]
    w = state["weight"]
    key = torch.where(ok & ~torch.isnan(w), w, low).double()
    key = torch.where((t < c["first"]) | (t >= lens - c["last"]), math.inf, key)
    # behind every token of the prefix, whatever its weight: sort by (inside, key), ties by index
    at = torch.sort(key, dim=1, descending=True, stable=True).indices
    at = at.gather(1, torch.sort((at < lens).to(torch.int8), dim=1, descending=True, stable=True).indices)
    kept = torch.where(t < new, at, rows).sort(1).values      # ascending; `rows` marks the end
    live = kept < rows
    src = torch.where(live, kept, 0)
    full = torch.zeros((c["n"], rows - cap), dtype=torch.bool, device=dev)
    live32 = torch.cat([live, full], 1)
    src32 = torch.cat([src, torch.zeros_like(full, dtype=src.dtype)], 1)
    index = src32[:, None, None, None, :, None].expand(-1, c["layers"], 2, c["kvh"], -1, c["hd"])
    x = codes.gather(4, index).view(torch.float8_e4m3fn).float() * sc.gather(4, (src32 // BLOCK)[:, None, None, None, :].expand(index.shape[:-1]))[..., None]
    x = torch.where(live32[:, None, None, None, :, None], x, torch.zeros((), device=dev))
    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros((), device=dev)).unflatten(4, (-1, BLOCK)).amax((-1, -2))
    s = block_scale(a)
    q = codes_of(x, s.repeat_interleave(BLOCK, 4)[..., None])
    to_codes.copy_(torch.where(live32[:, None, None, None, :, None], q, to_codes))
    blk = live32[:, ::BLOCK]
    to_sc.copy_(torch.where(blk[:, None, None, None, :], s, to_sc))
    to_words.copy_(torch.where(blk, pack_bits(live32 & seen(c, state["lens"], words).gather(1, src32)), to_words))
    state["weight_out"].copy_(torch.where(live, w.gather(1, src), state["weight_out"]))
    state["kept"].copy_(torch.where(live, kept.to(torch.int32), state["kept"]))


# ---- what a program has in hand ----------------------------------------------------------------------------------------

def _planes(c, g, n, dtype, rows):
    """Planes as a backbone gives them: heads of different size, a few large channels, a first token that stands out."""
    d, dev = c["kvh"] * c["hd"], g.device
    x = torch.randn((n, c["layers"], 2, rows, d), generator=g, device=dev, dtype=torch.float32)
    x *= torch.exp(0.4 * torch.randn((1, c["layers"], 2, 1, d), generator=g, device=dev))
    x[:, :, :, :1] *= 3.0
    return x.to(DT[dtype])


def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    rows, _, _, _, nbytes = sizes(c)
    lens = lengths(c, seed)
    n = c["n"]
    visible = torch.rand((n, rows), generator=g, device=dev) >= c["hide"]
    if c["hide"] > 0.5:
        visible[::5] = False     # environments that see nothing
    state = {"case": c, "layout": (c["layers"], c["kvh"], c["hd"], c["cap"]), "lens": lens,
             "pool": torch.zeros((n, nbytes), dtype=torch.uint8, device=dev), "layer": c["layers"] - 1}
    if c["op"] == "quantize":
        state["planes"] = _planes(c, g, n, c["dtype"], c["cap"])
        state["mask"] = visible[:, :c["cap"]].to(torch.uint8).contiguous() if c["hide"] else None
        return state
    step = max(1, int(2e8 / (rows * 2 * c["layers"] * c["kvh"] * c["hd"])))
    for i in range(0, n, step):
        x = _planes(c, g, min(step, n - i), "bf16", rows).float()
        plain_quantize(c, state["pool"][i:i + step], x, lens[i:i + step], visible[i:i + step])
    if c["op"] == "evict":
        state["dst"] = torch.zeros_like(state["pool"])
        state["weight"] = torch.rand((n, c["cap"]), generator=g, device=dev) ** 4
        state["weight_out"] = torch.zeros_like(state["weight"])
        state["kept"] = torch.zeros((n, c["cap"]), dtype=torch.int32, device=dev)
        state["keep"] = torch.full((n,), c["keep"], dtype=torch.int32)
        return state
    # queries: a few components that favour some tokens, so that the weights are neither flat nor a single one
    state["q"] = (1.3 * torch.randn((n, c["H"], c["kvh"] * c["G"], c["hd"]), generator=g, device=dev)).to(DT[c["dtype"]])
    if c["op"] == "weigh":
        state["lse"] = plain_attend(c, state)[1]
        state["weight"] = torch.rand((n, c["cap"]), generator=g, device=dev)
    return state


def run(state):
    c = state["case"]
    if own:
        from paper_2609_27547_b200 import prefix8
        lay = prefix8.Layout(*state["layout"])
    if c["op"] == "quantize":
        if own:
            prefix8.quantize(lay, state["pool"], state["planes"], state["lens"], mask=state["mask"])
        else:
            x = state["planes"].float()
            rows = sizes(c)[0]
            x = torch.nn.functional.pad(x, (0, 0, 0, rows - c["cap"]))
            visible = torch.ones((c["n"], rows), dtype=torch.bool, device=x.device)
            if state["mask"] is not None:
                visible[:, :c["cap"]] = state["mask"] != 0
            plain_quantize(c, state["pool"], x, state["lens"], visible)
        codes, scales, words = views(c, state["pool"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales, "mask": words}
    if c["op"] == "attend":
        if own:
            out, lse = prefix8.attend(lay, state["pool"], state["q"], state["lens"], layer=state["layer"])
        else:
            out, lse = plain_attend(c, state)
        return {"out": out, "lse": lse}
    if c["op"] == "weigh":
        if own:
            prefix8.weigh(lay, state["pool"], state["q"], state["lse"], state["lens"], state["weight"], layer=state["layer"], accumulate=c["add"])
        else:
            plain_weigh(c, state)
        return {"weight": state["weight"]}
    if own:
        prefix8.evict(lay, state["pool"], state["dst"], state["weight"], state["lens"], state["keep"], protect_first=c["first"],
                      protect_last=c["last"], weight_out=state["weight_out"], kept=state["kept"])
    else:
        plain_evict(c, state)
    codes, scales, words = views(c, state["dst"])
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales, "mask": words, "kept": state["kept"], "weight": state["weight_out"]}


# ---- the definitions in 64 bits, one environment at a time -----------------------------------------------------------

E4M3 = None


def table():
    """The values that the e4m3 codes 0 .. 126 stand for, in order."""
    global E4M3
    if E4M3 is None:
        v = [(k % 8) * 2.0 ** -9 if k < 8 else (1 + (k % 8) / 8) * 2.0 ** (k // 8 - 7) for k in range(127)]
        E4M3 = torch.tensor(v, dtype=torch.float64, device="cuda")
    return E4M3


def nearest(y):
    """The e4m3 value next to y (64 bits, no NaN), ties to the even code, saturated."""
    t = table()
    a = y.abs().clamp_max(448.0)
    hi = torch.searchsorted(t, a).clamp_max(126)
    lo = (hi - 1).clamp_min(0)
    up, down = t[hi] - a, a - t[lo]
    k = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(t[k], y)


def encode(x, groups):
    """x [rows, cols] in 64 bits and which rows make a block -> (values of the codes, the blocks' scales)."""
    amax = torch.zeros(int(groups[-1]) + 1, dtype=torch.float64, device=x.device).scatter_reduce(0, groups, x.abs().amax(1), "amax")
    s = torch.where(amax > 0, torch.exp2(torch.ceil(torch.log2(amax.clamp_min(1e-300) / 448.0))), 1.0)
    # the quotient has to lie in (224, 448]: put right what the logarithm's last bit got wrong
    s = torch.where((amax > 0) & (amax / s > 448.0), 2 * s, torch.where((amax > 0) & (amax / s <= 224.0), s / 2, s))
    return nearest(x / s[groups][:, None]), s


def exact(c, seed):
    state = prepare(c, seed)
    rows, _, _, _, _ = sizes(c)
    n, dev = c["n"], "cuda"
    if n * c["layers"] * 2 * c["kvh"] > 9000 and c["op"] in ("quantize", "evict"):
        return None
    codes, sc, words = views(c, state["pool"])
    lens = state["lens"].tolist()
    vis = [[(int(w) >> b) & 1 for w in row for b in range(BLOCK)] for row in words.cpu().tolist()]
    if c["op"] in ("quantize", "evict"):
        o_codes = torch.zeros(codes.shape, dtype=torch.float64, device=dev)
        o_sc = torch.zeros(sc.shape, dtype=torch.float64, device=dev)
        o_w = state["weight_out"].double() if c["op"] == "evict" else None
        for i in range(n):
            if c["op"] == "quantize":
                take = list(range(lens[i]))
                hidden = [False] * lens[i] if state["mask"] is None else (state["mask"][i, :lens[i]] == 0).tolist()
            else:
                w = state["weight"][i].tolist()
                rank = []
                for t in range(lens[i]):
                    guard = t < c["first"] or t >= lens[i] - c["last"]
                    rank.append((0 if guard else 1, 0.0 if guard else -(w[t] if vis[i][t] else -math.inf), t))
                take = sorted(r[2] for r in sorted(rank)[:min(c["keep"], lens[i])])
                hidden = [False] * len(take)
                o_w[i, :len(take)] = state["weight"][i, take].double()
            if not take:
                continue
            k = len(take)
            idx = torch.tensor(take, device=dev)
            off = torch.tensor(hidden, device=dev)
            groups = torch.arange(k, device=dev) // BLOCK
            for layer in range(c["layers"]):
                for plane in range(2):
                    for h in range(c["kvh"]):
                        if c["op"] == "quantize":
                            x = state["planes"][i, layer, plane, :k, h * c["hd"]:(h + 1) * c["hd"]].double()
                        else:
                            x = decode(codes[i, layer, plane, h][idx]) * sc[i, layer, plane, h][idx // BLOCK].double()[:, None]
                        x = x.masked_fill(off[:, None], 0.0)
                        o_codes[i, layer, plane, h, :k], o_sc[i, layer, plane, h, :int(groups[-1]) + 1] = encode(x, groups)
        out = {"codes": o_codes, "scales": o_sc, "mask": None}
        return out if c["op"] == "quantize" else {**out, "kept": None, "weight": o_w}
    heads = c["kvh"] * c["G"]
    out = torch.zeros((n, c["H"], heads, c["hd"]), dtype=torch.float64, device=dev)
    lse = torch.full((n, c["H"], heads), -math.inf, dtype=torch.float64, device=dev)
    weight = state["weight"].double() if c["op"] == "weigh" else None
    for i in range(n):
        if c["op"] == "weigh" and not c["add"]:
            weight[i, :lens[i]] = 0.0
        see = torch.tensor([t for t in range(lens[i]) if vis[i][t]], device=dev, dtype=torch.int64)
        if not see.numel():
            continue
        kv = decode(codes[i, state["layer"]][:, :, see]) * sc[i, state["layer"]][:, :, see // BLOCK].double()[..., None]
        kv = kv.repeat_interleave(c["G"], 1)                                  # [2, heads, tokens, hd]
        s = torch.einsum("hnd,ntd->nht", state["q"][i].double(), kv[0]) / math.sqrt(c["hd"])
        if c["op"] == "weigh":
            weight[i, see] += torch.exp(s - state["lse"][i].double().t()[..., None]).sum((0, 1))
        else:
            lse[i] = torch.logsumexp(s, -1).t()
            out[i] = torch.einsum("nht,ntd->hnd", torch.softmax(s, -1), kv[1])
    return {"weight": weight} if c["op"] == "weigh" else {"out": out, "lse": lse}


def decode(codes):
    """e4m3 codes (uint8, no NaN) -> values in 64 bits."""
    return torch.where(codes >= 128, -1.0, 1.0) * table()[(codes & 127).long().clamp_max(126)]
