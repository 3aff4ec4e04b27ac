"""What the operators on paged caches are measured on.

A paged cache keeps the keys and values of many sequences (observation histories of environments) in pages of a fixed number of
tokens.  A page holds, for all layers, [kv_layers][2][kv_heads][page_tokens][head_dim] elements (keys, then values; bf16 or fp32) and
one bit per token that says whether queries may see it.  A pool is a uint8 tensor [n_pages, page_bytes]; a table
(int32 [n, width], on the device) names the pages of each sequence.  Four operators work on it, and a host-side book that knows which
page belongs to whom:

  append  the keys and values of new tokens -> pages
  attend  attention of a chunk of new tokens (one token, or thousands) over the whole sequence
  copy    pages to other pages: what a fork needs before its first own token, and what compaction moves
  gather  pages -> planes [kv_layers][2][P][kv_heads * head_dim], as the action head takes them
"""
import math

import torch

own = False

WORD = 32
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the page, and the cases ------------------------------------------------------------------------------------------

def page(c):
    """(elements, bytes of them, mask words, bytes of a page)"""
    elems = c["layers"] * 2 * c["kvh"] * c["T"] * c["hd"]
    nb = elems * (4 if c["dtype"] == "f32" else 2)
    return elems, nb, c["T"] // WORD, -(-(nb + c["T"] // 8) // 128) * 128


def views(c, pool):
    """(elements [n_pages, layers, 2, kvh, T, hd], mask words [n_pages, T / 32]) of a pool."""
    _, nb, w, _ = page(c)
    return (pool[:, :nb].view(DT[c["dtype"]]).unflatten(1, (c["layers"], 2, c["kvh"], c["T"], c["hd"])),
            pool[:, nb:nb + 4 * w].view(torch.int32))


def lengths(c, seed):
    """(lengths with the new tokens, numbers of new tokens), on the host: the same ones for each seed, dealt out anew."""
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(c["lo"], c["len"] + 1, (c["n"],), generator=g, dtype=torch.int32)
    lens[-1] = c["len"]
    new = torch.randint(c.get("new_lo", 0), c.get("new", 0) + 1, (c["n"],), generator=g, dtype=torch.int32)
    if c.get("single"):      # so many of the sequences add one token only
        new[torch.rand(c["n"], generator=g) < c["single"]] = 1
    order = torch.randperm(c["n"], generator=torch.Generator().manual_seed(seed * 2 + 1))
    return lens[order], torch.minimum(new, lens)[order]


def wide(c):
    """Columns of the tables of sequences after a fork or a compaction."""
    return -(-(c["len"] + 1) // c["T"])


def listed():
    def case(name, op, n, lo, length, kvh, hd, T, **kw):
        return dict(dict(name=name, op=op, n=n, lo=lo, len=length, kvh=kvh, hd=hd, T=T, layers=1, dtype="bf16"), **kw)
    return [
        # one robot's next token: latency
        case("attend_one_token", "attend", 1, 256, 256, 16, 64, 64, G=1, new_lo=1, new=1, causal=True, window=0, hide=0.0),
        # a batch of environments decodes one token each, four query heads on each key/value head
        case("attend_decode_group", "attend", 192, 512, 2048, 4, 128, 64, G=4, new_lo=1, new=1, causal=True, window=0, hide=0.0),
        # one long history takes in a short observation
        case("attend_long_history", "attend", 2, 60001, 65537, 4, 128, 128, G=4, new_lo=8, new=8, causal=True, window=0, hide=0.0),
        # a mixed batch: half decode, half bring ragged chunks, padded camera tokens are hidden
        case("attend_mixed", "attend", 64, 200, 1500, 8, 64, 32, G=2, new_lo=2, new=300, single=0.5, causal=True, window=0, hide=0.1),
        # the small fp32 model: observations whose tokens see one another
        case("attend_observation_f32", "attend", 96, 64, 512, 4, 64, 32, G=1, new_lo=16, new=64, causal=False, window=0, hide=0.0, dtype="f32"),
        # long chunks of a prefill over what is there already
        case("attend_chunk_large", "attend", 4, 8192, 16384, 4, 128, 128, G=4, new_lo=2000, new=2048, causal=True, window=0, hide=0.0),
        # every environment of a group adds one token
        case("append_one_token", "append", 64, 100, 900, 16, 64, 64, new_lo=1, new=1, hide=0.0),
        # the observations of a group of the large bf16 head: slices of one fused projection, padded camera tokens hidden
        case("append_group", "append", 128, 700, 1024, 16, 128, 64, new_lo=200, new=256, hide=0.1),
        # rollouts branch off: every history gets children, which share its full pages and copy the one they will write to
        case("copy_fork", "copy", 64, 100, 700, 8, 64, 64, layers=2, kids=7),
        # every other sequence was reset: the pages that are left move together
        case("copy_compact", "copy", 256, 500, 900, 16, 64, 64, drop=2),
        # one environment's history goes to the small fp32 head
        case("gather_one_f32", "gather", 1, 256, 256, 4, 64, 32, layers=2, dtype="f32", hide=0.0),
        # a group's histories go to the large bf16 head
        case("gather_group", "gather", 128, 700, 768, 16, 128, 64, hide=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "attend", "append", "copy", "gather"])
    hd, kvh, T = rng.choice([32, 64, 64, 128, 128]), rng.choice([1, 2, 4, 8, 16]), rng.choice([32, 64, 128, 256])
    dtype, layers = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([1, 1, 2])
    length = _log(rng, 1, 4000) if rng.random() < 0.8 else _log(rng, 4000, 60000)
    room = {"attend": 200e6, "append": 120e6, "gather": 120e6, "copy": 60e6}[op]
    n = _log(rng, 1, max(1, min(int(room / (2 * layers * kvh * hd * length)), 400)))
    c = dict(op=op, n=n, lo=rng.choice([1, length // 2 + 1, length]), len=length, kvh=kvh, hd=hd, T=T, layers=layers, dtype=dtype)
    if op == "copy":
        c["n"] = n = max(n, 2)
        if rng.random() < 0.5:
            c["kids"] = max(1, min(rng.randint(1, 8), int(400e6 / (2 * layers * kvh * hd * T * n))))
        else:
            c["drop"] = rng.choice([2, 3])
        return c
    c["hide"] = rng.choice([0.0, 0.0, 0.1, 0.6])
    if op == "attend":
        c["G"] = rng.choice([1, 1, 2, 3, 4, 8])
        c["new"] = rng.choice([1, rng.randint(1, 16), _log(rng, 1, 300), _log(rng, 1, 2048)])
        c["new"] = min(c["new"], length)
        # the pairs of a query and a token: 4 hd operations for each
        most = (1.6e11 if dtype == "bf16" else 2e10) / hd
        while n * c["new"] * c["G"] * kvh * length > most and c["new"] * c["G"] * n > 1:
            if c["new"] > 1:
                c["new"] = c["new"] // 2
            elif c["G"] > 1:
                c["G"] = 1
            else:
                c["n"] = n = max(1, n // 2)
        c["new_lo"] = rng.choice([1, c["new"]])
        c["single"] = rng.choice([0.0, 0.0, 0.5])
        c["causal"] = rng.random() < 0.7
        c["window"] = rng.choice([0, 0, _log(rng, 1, length)]) if c["causal"] else 0
    elif op == "append":
        c["new"] = min(length, rng.choice([1, _log(rng, 1, 2048)]))
        c["new_lo"] = rng.choice([0, c["new"]])
    return c


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    d = c["kvh"] * c["hd"]
    lens, new = (x.double() for x in lengths(c, 0))
    if c["op"] == "append":
        t = float(new.sum())
        return {"bytes": t * 2 * d * e * 2, "flops": t * 2 * d}
    if c["op"] == "gather":
        t = float(lens.sum())
        return {"bytes": t * 2 * c["layers"] * d * e * 2, "flops": t * 2 * c["layers"] * d}
    if c["op"] == "copy":
        if "kids" in c:
            t = float((lens % c["T"]).sum()) * c["kids"]      # the filled part of the last page
        else:
            pages = torch.ceil(lens / c["T"])
            gone = float(pages[::c["drop"]].sum())
            t = gone * (1 - gone / float(pages.sum())) * c["T"]   # so many of the pages above the new end are alive
        return {"bytes": t * 2 * c["layers"] * d * e * 2, "flops": t * 2 * c["layers"] * d}
    heads = c["kvh"] * c["G"]
    if c["causal"]:
        w = lens if not c["window"] else torch.clamp(lens, max=c["window"])
        # query j of `new` sees min(len - new + 1 + j, window) tokens
        first = lens - new + 1
        full = torch.clamp(lens - torch.maximum(first, w) + 1, min=0)        # queries that see w tokens
        part = new - full
        pairs = float((full * w + part * (first + (part - 1) / 2)).sum())
        tokens = float(torch.minimum(lens, new - 1 + w).sum())
    else:
        pairs, tokens = float((lens * new).sum()), float(lens.sum())
    return {"bytes": 2 * tokens * d * e + float(new.sum()) * heads * (2 * c["hd"] * e + 4), "flops": 4.0 * heads * c["hd"] * pairs}


# ---- plain forms -------------------------------------------------------------------------------------------------------

def unpack(words, T):
    """[.., T / 32] words -> [.., T] truth values."""
    t = torch.arange(T, device=words.device)
    return ((words[..., t // WORD] >> (t % WORD).to(torch.int32)) & 1) == 1


def pack(bits):
    w = (bits.unflatten(-1, (-1, WORD)).to(torch.int64) << torch.arange(WORD, device=bits.device)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def places(c, state):
    """(page, slot in it) of every new token, in the order of the packed rows."""
    lens, new = state["lens"].long().cuda(), state["new"].long().cuda()
    seq = torch.repeat_interleave(torch.arange(c["n"], device=lens.device), new)
    first = torch.cumsum(new, 0) - new
    pos = torch.arange(seq.numel(), device=lens.device) - first[seq] + lens[seq] - new[seq]
    return state["table"][seq, pos // c["T"]].long(), pos % c["T"]


def plain_append(c, state):
    elems, words = views(c, state["pool"])
    pg, slot = places(c, state)
    see = torch.ones(pg.shape, dtype=torch.bool, device=pg.device) if state["mask"] is None else state["mask"] != 0
    bits = unpack(words, c["T"])
    bits[pg, slot] = see
    for p, x in enumerate((state["k"], state["v"])):
        elems[pg, state["layer"], p, :, slot] = torch.where(see[:, None, None], x, torch.zeros((), dtype=x.dtype, device=x.device))
    words.copy_(pack(bits))
    return {"elements": elems, "mask": words}


def plain_attend(c, state):
    elems, words = views(c, state["pool"])
    q, G, hd, layer = state["q"], c["G"], c["hd"], state["layer"]
    heads = c["kvh"] * G
    out = torch.zeros((q.shape[0], heads, hd), dtype=q.dtype, device=q.device)
    lse = torch.zeros((q.shape[0], heads), dtype=torch.float32, device=q.device)
    at = 0
    for i, (n, m) in enumerate(zip(state["lens"].tolist(), state["new"].tolist())):
        if m == 0:
            continue
        lo = max(0, n - m + 1 - c["window"]) // c["T"] if c["window"] else 0      # pages that no query's window reaches are left out
        pages = state["table"][i, lo:-(-n // c["T"])].long()
        kv = elems[pages, layer].permute(1, 2, 0, 3, 4).flatten(2, 3).float()       # [2, kvh, tokens, hd]
        pos = torch.arange(lo * c["T"], lo * c["T"] + kv.shape[2], device=q.device)
        ok = unpack(words[pages], c["T"]).flatten() & (pos < n)
        kv = torch.where(ok[None, None, :, None], kv, torch.zeros((), device=q.device))
        ok = ok[None].expand(m, -1)
        if c["causal"]:
            me = torch.arange(n - m, n, device=q.device)[:, None]
            ok = ok & (pos <= me)
            if c["window"]:
                ok = ok & (pos > me - c["window"])
        x = q[at:at + m].float().unflatten(1, (c["kvh"], G)).permute(1, 2, 0, 3).reshape(c["kvh"], G * m, hd)
        s = (x @ kv[0].transpose(1, 2) * (1.0 / math.sqrt(hd))).unflatten(1, (G, m))
        s = torch.where(ok, s, torch.full((), -math.inf, device=q.device))
        top = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
        s = torch.exp(s - top)
        z = s.sum(-1, keepdim=True)
        o = (s.flatten(1, 2) @ kv[1]).unflatten(1, (G, m)) / torch.where(z > 0, z, torch.ones_like(z))
        out[at:at + m] = o.permute(2, 0, 1, 3).flatten(1, 2).to(q.dtype)
        lse[at:at + m] = (top + torch.log(z)).squeeze(-1).permute(2, 0, 1).flatten(1, 2)
        at += m
    return {"out": out, "lse": lse}


def plain_gather(c, state):
    elems, words = views(c, state["pool"])
    planes, seen = state["planes"], state["seen"]
    for i, n in enumerate(state["lens"].tolist()):
        pages = state["table"][i, :-(-n // c["T"])].long()
        ok = unpack(words[pages], c["T"]).flatten()[:n]
        x = elems[pages].permute(1, 2, 0, 4, 3, 5).flatten(2, 3)[:, :, :n]           # [layers, 2, n, kvh, hd]
        x = torch.where(ok[:, None, None], x, torch.zeros((), dtype=x.dtype, device=x.device))
        planes[i, :, :, :n] = x.flatten(3)
        seen[i, :n] = ok.to(torch.uint8)
    return {"planes": planes, "seen": seen}


def plain_fork(c, state):
    """Children share their parent's full pages; the page that their next token falls into is copied to the lowest free one."""
    elems, words = views(c, state["pool"])
    T, free = c["T"], list(state["free"])
    src, dst, rows = [], [], []
    for i, n in enumerate(state["lens"].tolist()):
        for k in range(c["kids"]):
            row = state["rows"][i][:]
            if n % T == 0:
                row.append(free.pop(0))
            elif n % T:
                src.append(row[-1])
                dst.append(free.pop(0))
                row[-1] = dst[-1]
            rows.append((row, n))
    if src:
        a, b = torch.tensor(src, device=elems.device), torch.tensor(dst, device=elems.device)
        part = torch.tensor([n % T for row, n in rows if n % T], device=elems.device)
        inside = torch.arange(T, device=elems.device) < part[:, None]
        elems[b] = torch.where(inside[:, None, None, None, :, None], elems[a], elems[b])
        words[b] = pack(torch.where(inside, unpack(words[a], T), unpack(words[b], T)))
    table = torch.tensor([row + [-1] * (wide(c) - len(row)) for row, _ in rows], dtype=torch.int32)
    return {"elements": elems, "mask": words, "table": table}


def plain_compact(c, state):
    """The sequences that stay: their pages with the highest numbers move to the lowest free ones."""
    elems, words = views(c, state["pool"])
    T = c["T"]
    keep = [(row, n) for i, (row, n) in enumerate(zip(state["rows"], state["lens"].tolist())) if i % c["drop"]]
    used = sorted(p for row, _ in keep for p in row)
    holes = sorted(set(range(len(used))) - set(used))
    to = dict(zip(sorted((p for p in used if p >= len(used)), reverse=True), holes))
    fill = {p: min(T, n - j * T) for row, n in keep for j, p in enumerate(row)}
    if to:
        a, b = torch.tensor(list(to), device=elems.device), torch.tensor(list(to.values()), device=elems.device)
        inside = torch.arange(T, device=elems.device) < torch.tensor([fill[p] for p in to], device=elems.device)[:, None]
        elems[b] = torch.where(inside[:, None, None, None, :, None], elems[a], elems[b])
        words[b] = pack(torch.where(inside, unpack(words[a], T), unpack(words[b], T)))
    table = torch.tensor([[to.get(p, p) for p in row] + [-1] * (wide(c) - len(row)) for row, _ in keep], dtype=torch.int32)
    return {"elements": elems, "mask": words, "table": table}


# ---- what a program has in hand ----------------------------------------------------------------------------------------

def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    lens, new = lengths(c, seed)
    T, n = c["T"], c["n"]
    _, _, _, nbytes = page(c)
    counts = (-(-lens.long() // T)).tolist()
    used = sum(counts)
    spare = n * c["kids"] if "kids" in c else 3
    if c["op"] == "copy":
        # what a book has handed out: sequences grew in turn, lowest page first
        rows, at = [[] for _ in range(n)], 0
        for j in range(max(counts)):
            for i in range(n):
                if j < counts[i]:
                    rows[i].append(at)
                    at += 1
    else:
        order = torch.randperm(used + spare, generator=torch.Generator().manual_seed(seed)).tolist()
        rows = [[order.pop() for _ in range(k)] for k in counts]
    width = max(counts)
    table = torch.tensor([row + [-1] * (width - len(row)) for row in rows], dtype=torch.int32)
    state = {"case": c, "lens": lens, "new": new, "table": table.to(dev), "layer": c["layers"] - 1, "pool": torch.empty((used + spare, nbytes), dtype=torch.uint8, device=dev)}
    # keys and values as a backbone gives them: channels of different size, a first token that stands out; old data in rows that no sequence fills
    elems, words = views(c, state["pool"])
    size = torch.exp(0.4 * torch.randn((c["layers"], 2, c["kvh"], 1, c["hd"]), generator=g, device=dev))
    step = max(1, int(1e8 / page(c)[0]))
    for i in range(0, used + spare, step):
        x = torch.randn(elems[i:i + step].shape, generator=g, device=dev)
        elems[i:i + step] = (x * size).to(elems.dtype)
    see = torch.rand((used + spare, T), generator=g, device=dev) >= c.get("hide", 0.0)
    if c.get("hide", 0.0) > 0.5:
        see[table[4::5][table[4::5] >= 0].long().to(dev)] = False       # sequences that see nothing
    words.copy_(pack(see))
    if c["op"] == "copy":
        state["rows"] = rows
        state["free"] = list(range(used, used + spare))
        if own:     # a program has its book
            from paper_2609_27547_b200 import pages
            book = pages.Book(used + spare, T, n * (1 + c.get("kids", 0)))
            for j in range(max(counts)):
                some = [i for i in range(n) if j < counts[i]]
                book.extend(some, [min(int(lens[i]), (j + 1) * T) for i in some])
            state["book"] = book
        return state
    if c["op"] == "gather":
        state["planes"] = torch.zeros((n, c["layers"], 2, c["len"], c["kvh"] * c["hd"]), dtype=DT[c["dtype"]], device=dev)
        state["seen"] = torch.zeros((n, c["len"]), dtype=torch.uint8, device=dev)
        return state
    total = int(new.sum())
    if c["op"] == "append":
        # keys and values stand behind the queries in the rows of one projection
        qkv = (torch.randn((total, 3 * c["kvh"], c["hd"]), generator=g, device=dev) * 1.2).to(DT[c["dtype"]])
        state["k"], state["v"] = qkv[:, c["kvh"]:2 * c["kvh"]], qkv[:, 2 * c["kvh"]:]
        state["mask"] = (torch.rand(total, generator=g, device=dev) >= c["hide"]).to(torch.uint8) if c["hide"] else None
        return state
    state["q"] = (1.3 * torch.randn((total, c["kvh"] * c["G"], c["hd"]), generator=g, device=dev)).to(DT[c["dtype"]])
    return state


def run(state):
    c = state["case"]
    if own:
        from paper_2609_27547_b200 import pages
        lay = pages.Layout(c["layers"], c["kvh"], c["hd"], c["T"], DT[c["dtype"]])
    if c["op"] == "append":
        if not own:
            return plain_append(c, state)
        pages.append(lay, state["pool"], state["table"], state["k"], state["v"], state["new"], state["lens"], layer=state["layer"], mask=state["mask"])
    elif c["op"] == "attend":
        if not own:
            return plain_attend(c, state)
        out, lse = pages.attend(lay, state["pool"], state["table"], state["q"], state["new"], state["lens"], layer=state["layer"],
                                causal=c["causal"], window=c["window"])
        return {"out": out, "lse": lse}
    elif c["op"] == "gather":
        if not own:
            return plain_gather(c, state)
        pages.gather(lay, state["pool"], state["table"], state["lens"], state["planes"], mask=state["seen"])
        return {"planes": state["planes"], "seen": state["seen"]}
    else:
        if not own:
            return plain_fork(c, state) if "kids" in c else plain_compact(c, state)
        book, n = state["book"].clone(), c["n"]      # so that a pass finds the book as the one before it did
        if "kids" in c:
            kids = [n + i for i in range(n * c["kids"])]
            book.fork([i for i in range(n) for _ in range(c["kids"])], kids)
            moves = book.extend(kids, [v + 1 for v in state["lens"].tolist() for _ in range(c["kids"])])
            stay = kids
        else:
            book.shorten(list(range(0, n, c["drop"])), 0)
            moves = book.compact()
            stay = [i for i in range(n) if i % c["drop"]]
        pages.copy(lay, state["pool"], state["pool"], moves)
        elems, words = views(c, state["pool"])
        return {"elements": elems, "mask": words, "table": book.table(stay, wide(c))}
    elems, words = views(c, state["pool"])
    return {"elements": elems, "mask": words}


# ---- the definition in 64 bits, one sequence and head at a time --------------------------------------------------------

def exact(c, seed):
    if c["op"] != "attend":
        return None          # values are moved as they are: there is nothing to compute
    state = prepare(c, seed)
    lens, new = state["lens"].tolist(), state["new"].tolist()
    if work(c)["flops"] > 2.5e12 or sum(m > 0 for m in new) * c["kvh"] > 6000:
        return None
    elems, words = views(c, state["pool"])
    rows = state["table"].cpu().tolist()
    bits = words.cpu().tolist()
    q, T, G, dev = state["q"], c["T"], c["G"], "cuda"
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device=dev)
    at = 0
    for i in range(c["n"]):
        if new[i] == 0:
            continue
        see = [t for t in range(lens[i]) if (bits[rows[i][t // T]][t % T // WORD] >> (t % WORD)) & 1]
        if see:
            pos = torch.tensor(see, device=dev)
            pg = torch.tensor([rows[i][t // T] for t in see], device=dev)
            for h in range(c["kvh"]):
                k = elems[pg, state["layer"], 0, h, pos % T].double()
                v = elems[pg, state["layer"], 1, h, pos % T].double()
                for j0 in range(0, new[i], 256):
                    j1 = min(new[i], j0 + 256)
                    x = q[at + j0:at + j1, h * G:(h + 1) * G].double()
                    s = torch.einsum("jgd,td->jgt", x, k) / math.sqrt(c["hd"])
                    if c["causal"]:
                        back = torch.arange(lens[i] - new[i] + j0, lens[i] - new[i] + j1, device=dev)[:, None] - pos      # how far back a token lies
                        s = s.masked_fill(((back < 0) | ((back >= c["window"]) if c["window"] else False))[:, None], -math.inf)
                    l = torch.logsumexp(s, -1)
                    p = torch.where(l[..., None] > -math.inf, torch.exp(s - l[..., None]), 0.0)
                    lse[at + j0:at + j1, h * G:(h + 1) * G] = l
                    out[at + j0:at + j1, h * G:(h + 1) * G] = torch.einsum("jgt,td->jgd", p, v)
        at += new[i]
    return {"out": out, "lse": lse}
