"""Cases and plain forms of the paged KV cache of the routed attention stack, from the projections to the pages and back.

Operators that a serving loop runs one after another:

  rope     norms of query and key heads and the position rotation in one pass, rows to rows (what a prefill call takes)
  store    the same for a fused projection output, K and V rows put into the pages of their requests
  decode   one query row per request over its pages, each request dense (full attention) or sparse (sink + window) by its routing bit
  step     norms, rotation, storing of the newest token and the decode in one call
  pages    the pages themselves: finished requests released, beams forked, room reserved (a shared page that is about to be written is
           copied first), all on the device
  compact  the pages in use moved to the low end of the pool

Sizes: the head layouts (32/8, 28/4, 8/2), sinks, windows and context lengths of the benchmark's workloads.
"""
import math

import numpy as np
import torch

own = False     # False: the plain forms below; True: the framework's calls

DEV = "cuda:0"
D = 128         # head dimension
NONE = -1       # a table entry without a page
EPS = 1e-6


# ---- cases ------------------------------------------------------------------------------------------------------

def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _text(values):
    return ",".join(str(int(x)) for x in values)


def listed():
    llama = {"hq": 32, "hkv": 8}
    whole = {"rotary": 128, "style": "halves", "theta": 500000.0, "norm": True}
    return [
        # the projections of one decode step of a batch, far into their contexts (group of 7): latency of one launch
        {"name": "rope_tokens", "op": "rope", "hq": 28, "hkv": 4, "new": _text([1] * 24), "past": _text([5003 * i + 17 for i in range(24)]),
         "rotary": 64, "style": "pairs", "theta": 10000.0, "norm": True},
        # the rows of an admission batch, ragged, on their way into a prefill call
        {"name": "rope_prompts", "op": "rope", **llama, "new": "8192,777,6001,1500,300,4500,2160,1146", "past": "0,0,1000000,0,0,65536,0,0", **whole},
        # one decode step's tokens into their pages
        {"name": "store_tokens", "op": "store", **llama, "page": 16, "new": _text([1] * 32), "past": _text([(37 * i * i + 11 * i) % 2000 for i in range(32)]), **whole},
        # the prompts of an admission batch into their pages: bound by the memory
        {"name": "store_prompts", "op": "store", **llama, "page": 64, "new": "16384,777,6001,1500,300,4500,2160,1146", "past": "0,0,0,0,0,0,0,0", **whole},
        # a short chat, batch 1: latency of one launch
        {"name": "step_short", "op": "step", "hq": 8, "hkv": 2, "page": 16, "sink": 64, "window": 256, "modes": "1", "ctx": "333", **whole},
        # a large batch of short contexts: many small pieces of work
        {"name": "step_wide", "op": "step", **llama, "page": 16, "sink": 128, "window": 2048, "modes": "10" * 32,
         "ctx": _text([100 + (397 * i * i + 61 * i) % 3900 for i in range(64)]), **whole},
        # a single long context (group of 7), dense
        {"name": "decode_long", "op": "decode", "hq": 28, "hkv": 4, "page": 64, "sink": 128, "window": 4096, "modes": "1", "ctx": "131071"},
        # batched long-context decode, half of the requests sparse in this layer (what they do not need has been released)
        {"name": "decode_batch", "op": "decode", **llama, "page": 16, "sink": 128, "window": 4096, "modes": "11010010",
         "ctx": _text([65536 + 7 * i for i in range(8)])},
        # one step of a beam search: 8 groups of 4 beams, one group finished, the others reordered and given room for a token
        {"name": "pages_beams", "op": "pages", "hkv": 8, "page": 16, "slabs": 4, "pool": 4096, "beams": 4, "len": "100,257,1033,640,2047,48,3001,911", "more": 1},
        # an admission batch: finished requests go, prompts get their pages (per-layer pools of a group of 4 heads)
        {"name": "pages_admit", "op": "pages", "hkv": 4, "page": 16, "slabs": 2, "pool": 24576, "beams": 1,
         "len": "16384,0,6001,1500,12001,0,2160,0,300,4097,0,0,9000,0,0,777", "more": 8000},
        # a small pool after some requests have gone
        {"name": "compact_small", "op": "compact", "hkv": 2, "page": 16, "slabs": 2, "pool": 512, "len": "500,33,1200,16,815"},
        # a large pool, 60 % in use, prefixes shared: bound by the memory
        {"name": "compact_large", "op": "compact", "hkv": 8, "page": 32, "slabs": 2, "pool": 12000,
         "len": "65536,4096,20011,5003,30000,9999,30007,12288,7000,17000,4444,26000"},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    hq, hkv = rng.choice([(32, 8), (28, 4), (8, 2), (8, 8), (16, 1), (36, 3)])
    sink, window = rng.choice([(128, 4096), (128, 2048), (64, 256), (0, 500), (5, 33)])
    op = rng.choice(["rope", "store", "decode", "step", "pages", "compact"])
    page = rng.choice([16, 32, 64, 128])
    turn = {"rotary": rng.choice([128, 128, 64, 32, 96, 0]), "style": rng.choice(["halves", "pairs"]), "theta": rng.choice([1e4, 5e5, 1e6]), "norm": rng.random() < 0.7}
    if op in ("decode", "step"):
        b = _spread(rng, 1, 64)
        most = min(131072, (250000 if op == "decode" else 60000) // b)
        case = {"op": op, "hq": hq, "hkv": hkv, "page": page, "sink": sink, "window": window, "modes": "".join(rng.choice("01") for _ in range(b)),
                "ctx": _text(_spread(rng, 1, most) for _ in range(b))}
        return case if op == "decode" else {**case, **turn}
    if op in ("rope", "store"):
        room, new, past = 28000, [], []
        for _ in range(_spread(rng, 1, 48)):
            n = min(room, _spread(rng, 1, 9000)) if rng.random() < 0.95 else 0
            room -= n
            new.append(n)
            past.append(0 if rng.random() < 0.5 else _spread(rng, 1, 4096 if op == "store" else 2000000))
        new[0] = max(new[0], 1)
        return {"op": op, "hq": hq, "hkv": hkv, **({"page": page} if op == "store" else {}), "new": _text(new), "past": _text(past), **turn}
    lens = [_spread(rng, 1, 6000) if rng.random() < 0.9 else 0 for _ in range(_spread(rng, 2, 24))]
    beams = rng.choice([1, 2, 4, 5]) if op == "pages" else 1
    slabs = rng.choice([2, 4])
    held = sum(-(-n // page) for n in lens) + len(lens) * beams * 2
    more = _spread(rng, 1, 3000) if beams == 1 else 1
    pool = held + len(lens) * beams * (-(-more // page) + 1) + _spread(rng, 1, held)
    if op == "compact":
        return {"op": op, "hkv": hkv, "page": page, "slabs": slabs, "pool": pool, "len": _text(lens)}
    return {"op": op, "hkv": hkv, "page": page, "slabs": slabs, "pool": pool, "beams": beams, "len": _text(lens), "more": more}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _values(gen, rows, heads, spread):
    """Rows of a projection: unit noise whose channels differ in size (as those of keys do), a few of them large."""
    size = torch.exp(spread * torch.randn(heads, D, generator=gen, device=DEV))
    x = torch.empty(rows, heads, D, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    return x.mul_(size.to(torch.bfloat16))


def _dev(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _sum(values):
    return [0] + [int(x) for x in np.cumsum(values)]


def _pages(n, page):
    return -(-int(n) // page)


def _inv_freq(case):
    """Radians per position of every pair of rotated channels."""
    r = case["rotary"]
    return case["theta"] ** (-np.arange(0, r, 2, dtype=np.float64) / max(r, 1))


def _inputs(case, seed):
    """What the seed alone makes, on the device; index data on the host too."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 7919 + 13)
    host = np.random.default_rng([int(seed), 77])
    hkv, op = case["hkv"], case["op"]
    if op in ("pages", "compact"):
        s = _book(case, host)
        s["data"] = torch.empty(case["slabs"], case["pool"], case["page"], hkv, D, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
        return s
    hq = case["hq"]
    s = {}
    if op != "decode":
        s["weights"] = [(1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(torch.bfloat16) if case["norm"] else None for _ in "qk"]
    if op in ("rope", "store"):
        new, past = _ints(case["new"]), _ints(case["past"])
        s["new"], s["past"] = new, past
        held = [p + n if n else 0 for n, p in zip(new, past)]
    else:
        ctx = _ints(case["ctx"])
        new, held = [1] * len(ctx), ctx
        s["ctx"] = ctx
    # one fused projection output: query, key and value heads of a row beside one another
    s["qkv"] = torch.cat([_values(gen, sum(new), hq, 0.2), _values(gen, sum(new), hkv, 0.5), _values(gen, sum(new), hkv, 0.3)], 1)
    if op == "rope":
        return s
    # the pages of every request anywhere in the pool; a sparse request has kept those of its sink and its window
    page = case["page"]
    cols = max(_pages(n, page) for n in held)
    table = np.full((len(held), cols), NONE, dtype=np.int32)
    for b, n in enumerate(held):
        j = np.arange(_pages(n, page))
        if op != "store" and case["modes"][b] == "0":
            j = j[(j * page < case["sink"]) | ((j + 1) * page > n - case["window"])]
        table[b, j] = 0
    count = int((table == 0).sum())
    s["n_pages"] = count + 3
    table[table == 0] = host.permutation(s["n_pages"])[:count]
    s["table_host"] = table
    s["table"] = torch.from_numpy(table).to(DEV)
    if op == "store":
        s["k"], s["v"] = (torch.zeros(s["n_pages"], page, hkv, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    else:
        s["k"], s["v"] = (_values(gen, s["n_pages"] * page, hkv, x).reshape(s["n_pages"], page, hkv, D) for x in (0.5, 0.3))
    return s


def _book(case, host):
    """Tables and reference counts of a pool in use, and what the call is to do, on the host."""
    page, n_pages, beams = case["page"], case["pool"], case.get("beams", 1)
    lens = [n for n in _ints(case["len"]) for _ in range(beams)]
    more = case.get("more", 0)
    cols = _pages(max(lens) + more, page) + 1
    table = np.full((len(lens), cols), NONE, dtype=np.int32)
    free = iter(host.permutation(n_pages))
    for b, n in enumerate(lens):
        for j in range(_pages(n, page)):
            if b % beams and (j + 1) * page <= n:           # the beams of a group share all full pages
                table[b, j] = table[b - 1, j]
            elif beams == 1 and b and j < _pages(lens[b - 1], page) // 3 and b % 3 == 2:
                table[b, j] = table[b - 1, j]               # every third request shares a third of its neighbour's pages
            else:
                table[b, j] = next(free)
    refs = np.bincount(table[table >= 0], minlength=n_pages).astype(np.int32)
    s = {"table0": table, "refs0": refs}
    if case["op"] == "pages":
        gone = [b for b in range(len(lens)) if (b // beams) % 4 == 1]       # a quarter of the requests are done
        stay = [b for b in range(len(lens)) if b not in gone]
        s["gone"] = gone
        s["dst"] = [b for b in stay if beams > 1]
        s["src"] = [b - b % beams + int(host.integers(beams)) for b in s["dst"]]            # every beam goes on from one of its group
        s["rows"] = stay if beams > 1 else list(range(len(lens)))
        s["len"] = [0 if b in gone else lens[b] for b in s["rows"]]
        s["new_len"] = [n + more if beams > 1 or n == 0 else n + 1 for n in s["len"]]       # new prompts, or the next token
        s["fork_len"] = [lens[b] for b in s["dst"]]
    return s


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    op, hkv = case["op"], case["hkv"]
    if op in ("pages", "compact"):
        for name in ("table0", "refs0", "gone", "src", "dst", "fork_len", "rows", "len", "new_len"):
            if name in s:
                s[name] = torch.as_tensor(s[name], dtype=torch.int32).to(DEV)
        s["table"], s["refs"] = s["table0"].clone(), s["refs0"].clone()
        if op == "pages":
            s["begin"], s["end"] = torch.zeros_like(s["gone"]), torch.full_like(s["gone"], 2 ** 31 - 1)
    if op in ("rope", "store"):
        s["rows"], s["pos"] = _dev(_sum(s["new"])), _dev(s["past"])
        s["at"] = _dev(np.concatenate([p + np.arange(n) for n, p in zip(s["new"], s["past"])]))
        s["total"] = sum(s["new"])
    if op in ("decode", "step"):
        s["ctx_dev"] = _dev(s["ctx"])
        s["at"] = s["ctx_dev"] - 1
    if op != "decode" and op not in ("pages", "compact"):
        s["inv_freq"] = torch.from_numpy(_inv_freq(case)).to(DEV)
    if own:
        from paper_2604_07394_b200 import flux
        modes = case.get("modes") or "1" * max(len(s["new"]) if "new" in s else 1, 1)
        cfg = flux.make_config(1, case.get("hq", hkv), hkv, case.get("sink", 0), case.get("window", 1), len(modes), max(s.get("ctx", [1])) if "ctx" in s else 1 << 22)
        s["plan"] = flux.Plan(cfg, DEV)
        s["plan"].flux_router_apply(mask=np.array([[int(m)] for m in modes], dtype=np.uint8))
        if "inv_freq" in s:
            s["rope"] = flux.Rope(_inv_freq(case), q_weight=s["weights"][0], k_weight=s["weights"][1], eps=EPS, interleaved=case["style"] == "pairs", device=DEV)
        if op in ("store", "decode", "step"):
            s["pages"] = flux.Pages(s["k"], s["v"], s["table"])
        if op in ("pages", "compact"):
            s["pool"] = flux.PagePool(s["table"], s["refs"], list(s["data"]))
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------

def _heads(s):
    """Query, key and value rows of the fused projection output."""
    hq, hkv = s["case"]["hq"], s["case"]["hkv"]
    return s["qkv"][:, :hq], s["qkv"][:, hq:hq + hkv], s["qkv"][:, hq + hkv:]


def _turned(s, x, weight):
    """Norm of every head and rotation by the row's position, 32 bits (angles: 64)."""
    case, r = s["case"], s["case"]["rotary"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    if r == 0:
        return x
    angle = s["at"].double()[:, None] * s["inv_freq"][None, :]
    c, n = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    if case["style"] == "pairs":
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_rope(s):
    q, k, _ = _heads(s)
    return [_turned(s, q, s["weights"][0]).to(torch.bfloat16), _turned(s, k, s["weights"][1]).to(torch.bfloat16)]


def _put(s, request, k, v):
    """Rows into the pages of their requests, at the positions s["at"]."""
    page = s["case"]["page"]
    at = s["at"].long()
    row = s["table"][request, at // page].long() * page + at % page
    s["k"].view(-1, *s["k"].shape[2:])[row] = k.to(torch.bfloat16)
    s["v"].view(-1, *s["v"].shape[2:])[row] = v


def _plain_store(s):
    q, k, v = _heads(s)
    request = torch.bucketize(torch.arange(s["total"], device=DEV), s["rows"][1:].long(), right=True)
    _put(s, request, _turned(s, k, s["weights"][1]), v)
    return [_turned(s, q, s["weights"][0]).to(torch.bfloat16), s["k"], s["v"]]


def _attend(s, q):
    """softmax(q K^T / sqrt(D)) V over the kept positions of each request's pages, 32 bits."""
    case, hkv, page = s["case"], s["case"]["hkv"], s["case"]["page"]
    out = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
    for b, (n, m) in enumerate(zip(s["ctx"], case["modes"])):        # requests differ in length
        j = torch.arange(n, device=DEV)
        if m == "0" and n > case["sink"] + case["window"]:
            j = torch.cat([j[:case["sink"]], j[n - case["window"]:]])
        row = s["table"][b, j // page].long() * page + j % page
        k, v = (s[x].view(-1, hkv, D)[row].float() for x in "kv")
        g = q[b].float().reshape(hkv, -1, D)
        p = g @ k.permute(1, 2, 0) / math.sqrt(D)
        p = torch.exp(p - p.amax(-1, keepdim=True))
        out[b] = ((p @ v.transpose(0, 1)) / p.sum(-1, keepdim=True)).reshape(-1, D).to(torch.bfloat16)
    return out


def _plain_step(s):
    q, k, v = _heads(s)
    _put(s, torch.arange(len(s["ctx"]), device=DEV), _turned(s, k, s["weights"][1]), v)
    return [_attend(s, _turned(s, q, s["weights"][0])), s["k"], s["v"]]


def _count(s, pages, held, by):
    """Adds `by` to the reference counts of the held entries."""
    s["refs"].index_add_(0, pages.clamp(min=0).flatten(), (held.int() * by).flatten())


def _plain_release(s):
    table, page = s["table"], s["case"]["page"]
    cols = torch.arange(table.shape[1], device=DEV)
    rows, first = s["gone"].long(), (s["begin"].long() + page - 1) // page
    last = s["end"].long().clamp(max=table.shape[1] * page) // page
    old = table[rows]
    go = (cols >= first[:, None]) & (cols < last[:, None]) & (old >= 0)
    _count(s, old, go, -1)
    table[rows] = torch.where(go, NONE, old)


def _plain_fork(s):
    table, page = s["table"], s["case"]["page"]
    cols = torch.arange(table.shape[1], device=DEV)
    new, old = table[s["src"].long()], table[s["dst"].long()]
    new = torch.where(cols < ((s["fork_len"].long() + page - 1) // page)[:, None], new, NONE)
    _count(s, new, new >= 0, 1)
    _count(s, old, old >= 0, -1)
    table[s["dst"].long()] = new


def _plain_reserve(s):
    """The pages of positions len .. new_len - 1 become the row's own: free ones, lowest first, in the order of the rows; a shared page that
    is already begun is copied, unless all who share it are listed: then the last of them keeps it."""
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    rows, n0, n1 = s["rows"].long(), s["len"].long()[:, None], s["new_len"].long()[:, None]
    cols = torch.arange(table.shape[1], device=DEV)
    old = table[rows].long()
    want = (cols >= n0 // page) & (cols < (n1 + page - 1) // page) & (n1 > n0)
    at = old.clamp(min=0)
    shared = want & (old >= 0) & (refs[at] > 1)
    begun = shared & (cols == n0 // page) & (n0 % page != 0)
    writers = torch.zeros_like(refs).index_add_(0, at.flatten(), begun.int().flatten())
    place = torch.arange(len(rows), device=DEV)[:, None].expand_as(at)
    last = torch.full_like(refs, -1, dtype=torch.int64).scatter_reduce_(0, at.flatten(), torch.where(begun, place, -1).flatten(), "amax")
    need = want & ((old < 0) | (shared & ~(begun & (writers[at] == refs[at]) & (last[at] == place))))
    granted = need.sum(1).cumsum(0) <= (refs == 0).sum()
    need = need & granted[:, None]
    free = torch.argsort((refs != 0).int(), stable=True)
    page_of = free[(need.flatten().long().cumsum(0) - 1).clamp(min=0)].reshape(need.shape)
    new = torch.where(need, page_of, old)
    # one page of a row at most is copied, up to the row's length; the others write what a page in use holds to itself
    c = (n0 // page).clamp(max=table.shape[1] - 1)
    copy = (need & begun).gather(1, c)
    idle = refs.argmax()
    src, dst = (torch.where(copy, x.gather(1, c), idle)[:, 0] for x in (old, new))
    rowmask = copy & (torch.arange(page, device=DEV) < n0 % page)
    data = s["data"]
    data[:, dst] = torch.where(rowmask[None, :, :, None, None], data[:, src], data[:, dst])
    _count(s, old, need & shared, -1)
    _count(s, new, need, 1)
    table[rows] = new.int()
    return granted.int()


def _plain_pages(s):
    _plain_release(s)
    _plain_fork(s)
    granted = _plain_reserve(s)
    return [s["table"], s["refs"], granted, s["data"].view(torch.int16)]


def _plain_compact(s):
    table, refs, data = s["table"], s["refs"], s["data"]
    used, at = refs > 0, torch.arange(refs.numel(), device=DEV)
    count = used.sum()
    move = used & (at >= count)
    free = torch.argsort(used.int(), stable=True)
    order = (move.long().cumsum(0) - 1).clamp(min=0)
    goes = torch.where(move, free[order], at)
    comes = at.scatter_reduce(0, torch.where(move, goes, at), torch.where(move, at, NONE), "amax")      # the page whose content a page gets
    data.copy_(data[:, comes])
    there = torch.where(used, goes, NONE).int()
    table.copy_(torch.where(table >= 0, there[table.clamp(min=0).long()], NONE))
    refs.copy_(torch.where(at < count, refs[comes], 0))
    return [table, refs, there, count.int().reshape(1), data.view(torch.int16)]


def run(state):
    s, op = state, state["case"]["op"]
    if op in ("pages", "compact"):      # the same tables for every pass
        s["table"].copy_(s["table0"])
        s["refs"].copy_(s["refs0"])
    if not own:
        if op == "decode":
            return _attend(s, _heads(s)[0])
        return {"rope": _plain_rope, "store": _plain_store, "step": _plain_step, "pages": _plain_pages, "compact": _plain_compact}[op](s)
    plan = s["plan"]
    if op == "pages":
        plan.flux_pages_release(s["pool"], s["gone"], s["begin"], s["end"])
        plan.flux_pages_fork(s["pool"], s["src"], s["dst"], s["fork_len"])
        granted = plan.flux_pages_reserve(s["pool"], s["rows"], s["len"], s["new_len"])
        return [s["table"], s["refs"], granted, s["data"].view(torch.int16)]
    if op == "compact":
        there, count = plan.flux_pages_compact(s["pool"])
        return [s["table"], s["refs"], there, count, s["data"].view(torch.int16)]
    q, k, v = _heads(s)
    if op == "rope":
        return list(plan.flux_qk_norm_rope(s["rope"], q, k, s["at"]))
    if op == "store":
        return [plan.flux_paged_store(s["pages"], k, v, s["rows"], s["pos"], rope=s["rope"], q=q), s["k"], s["v"]]
    if op == "decode":
        return plan.flux_attn_decode_paged(0, len(s["ctx"]), q, s["pages"], s["ctx_dev"])
    return [plan.flux_attn_decode_step_paged(0, len(s["ctx"]), q, k, v, s["pages"], s["ctx_dev"], rope=s["rope"]), s["k"], s["v"]]


# ---- work and exact values --------------------------------------------------------------------------------------

def _kept(case, n, m):
    return n if m == "1" or n <= case["sink"] + case["window"] else case["sink"] + case["window"]


def work(case):
    hkv, op = case["hkv"], case["op"]
    if op in ("rope", "store"):      # rows in and out
        rows = sum(_ints(case["new"]))
        heads = case["hq"] + (2 if op == "store" else 1) * hkv
        return {"bytes": 2 * rows * heads * D * 2 + 4 * rows, "flops": 10 * rows * heads * D}
    if op in ("decode", "step"):
        ctx = _ints(case["ctx"])
        rows = sum(_kept(case, n, m) for n, m in zip(ctx, case["modes"]))
        entries = sum(_pages(_kept(case, n, m), case["page"]) for n, m in zip(ctx, case["modes"]))
        return {"bytes": 2 * hkv * rows * D * 2 + 4 * entries + 2 * len(ctx) * (case["hq"] + (2 * hkv if op == "step" else 0)) * D * 2, "flops": 4 * case["hq"] * D * rows}
    s = _book(case, np.random.default_rng([0, 77]))
    used = int((s["refs0"] > 0).sum())
    row = case["slabs"] * hkv * D * 2
    if op == "compact":             # what lies beyond the pages in use moves; entries and counts in and out
        moved = int((s["refs0"][used:] > 0).sum())
        return {"bytes": 2 * moved * case["page"] * row + 2 * 4 * int((s["table0"] >= 0).sum()) + 2 * 4 * case["pool"], "flops": 0}
    page, beams = case["page"], case["beams"]
    gone = int((s["table0"][s["gone"]] >= 0).sum())
    forked = sum(_pages(n, page) for n in s["fork_len"])
    fresh = sum(_pages(b, page) - _pages(a, page) for a, b in zip(s["len"], s["new_len"]))
    # of k beams that go on from one, k - 1 copy the rows of its begun page
    copies = sum(n % page for n, a, b in zip(s["fork_len"], s["src"], s["dst"]) if a in s["src"][:s["dst"].index(b)]) if beams > 1 else 0
    # entries taken out, put in and copied, their counts in and out; the counts up to the last free page that is taken
    return {"bytes": 4 * (3 * gone + 6 * forked + 3 * fresh) + 4 * fresh * 2 + 2 * copies * row, "flops": 0}


def _exact_turned(case, x, at, weight):
    """The same as a product of complex numbers, 64 bits."""
    r = case["rotary"]
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * weight.double()
    if r == 0:
        return x
    phase = torch.tensor(at, dtype=torch.float64, device=DEV)[:, None] * torch.from_numpy(_inv_freq(case)).to(DEV)
    turn = torch.polar(torch.ones_like(phase), phase)[:, None]
    y = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if case["style"] == "pairs" else (slice(0, r // 2), slice(r // 2, r))
    z = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    op, hkv = case["op"], case["hkv"]
    if op in ("pages", "compact"):
        return None
    x = _inputs(case, seed)
    hq = case["hq"]
    q, k, v = x["qkv"][:, :hq], x["qkv"][:, hq:hq + hkv], x["qkv"][:, hq + hkv:]
    if op in ("rope", "store"):
        at = [p + i for n, p in zip(x["new"], x["past"]) for i in range(n)]
        request = [b for b, n in enumerate(x["new"]) for _ in range(n)]
    else:
        at, request = [n - 1 for n in x["ctx"]], list(range(len(x["ctx"])))
    if op != "decode":
        q, k = _exact_turned(case, q, at, x["weights"][0]), _exact_turned(case, k, at, x["weights"][1])
    if op == "rope":
        return [q, k]
    page, table = case["page"], x["table_host"]
    if op != "decode":
        slot = torch.tensor([int(table[b, p // page]) * page + p % page for b, p in zip(request, at)], device=DEV)
        pools = []
        for pool, rows in ((x["k"], k), (x["v"], v)):
            y = pool.double().reshape(-1, hkv, D)
            y[slot] = rows.double()
            pools.append(y)
        whole = [p.reshape(-1, page, hkv, D) for p in pools]
        if op == "store":
            return [q, *whole]
        pools[0] = pools[0].to(torch.bfloat16).double()       # the cache holds the newest key in its own type
    else:
        pools = [x[z].reshape(-1, hkv, D) for z in "kv"]
    out = torch.empty(len(x["ctx"]), hq, D, dtype=torch.float64, device=DEV)
    for b, (n, m) in enumerate(zip(x["ctx"], case["modes"])):
        seen = [p for p in range(n) if m == "1" or p < case["sink"] or p >= n - case["window"]]
        p = np.array(seen)
        slot = torch.from_numpy(table[b, p // page].astype(np.int64) * page + p % page).to(DEV)
        for h in range(hq):
            kk, vv = (pool[:, h // (hq // hkv)][slot].double() for pool in pools)
            w = torch.softmax(kk @ q[b, h].double() / math.sqrt(D), 0)
            out[b, h] = w @ vv
    return [out, *whole] if op == "step" else out
