"""Cases and plain forms of the packed-prompt and 8-bit-cache operators of the routed attention stack.

Three operators that a serving loop runs one after another for each layer:

  prefill  causal attention of several requests' prompts (or prompt chunks) packed row after row, grouped heads, each
           request dense (full attention) or sparse (sink + window) by its routing bit
  store    the K / V rows of that layer put into per-request caches held in 8 bits, one scale for each block of 16
           positions and head (the newest, incomplete block stays in bf16), and read back as the values they stand for
  decode   one query row per request over such a cache

Sizes: the head layouts (32/8, 28/4, 8/2), sinks, windows and context lengths of the benchmark's workloads.
"""
import math

import numpy as np
import torch

own = False     # False: the plain forms below; True: the framework's calls

DEV = "cuda:0"
D = 128         # head dimension
BLOCK = 16      # positions that share one scale


# ---- cases ------------------------------------------------------------------------------------------------------

def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _text(values):
    return ",".join(str(int(x)) for x in values)


def listed():
    llama = {"hq": 32, "hkv": 8}
    return [
        # a handful of chat turns that arrive together: latency of one launch, lengths from one token up, an empty slot
        {"name": "prefill_short", "op": "prefill", "hq": 8, "hkv": 2, "sink": 64, "window": 256, "modes": "1010101010101010",
         "new": "1,17,64,200,0,129,33,128,7,300,96,2,150,65,31,255", "past": "0,0,0,0,0,0,0,0,0,0,0,0,0,0,0,0"},
        # an ordinary admission batch: documents of very different lengths, half of the requests routed to sparse
        {"name": "prefill_mixed", "op": "prefill", **llama, "sink": 128, "window": 2048, "modes": "10110100",
         "new": "4096,777,6001,1500,300,2500,64,1146", "past": "0,0,0,0,0,0,0,0"},
        # chunked prefill: the next chunk of long prompts whose earlier chunks are already cached (group of 7)
        {"name": "prefill_chunks", "op": "prefill", "hq": 28, "hkv": 4, "sink": 128, "window": 4096, "modes": "1001",
         "new": "2048,2048,1000,4096", "past": "16384,30000,0,8192"},
        # long prompts, all dense: bound by the matrix products
        {"name": "prefill_long", "op": "prefill", **llama, "sink": 128, "window": 4096, "modes": "1111",
         "new": "16384,8192,5000,3192", "past": "0,0,0,0"},
        # the prompts of an admission batch enter their caches
        {"name": "store_prompts", "op": "store", "fmt": "e4m3", **llama, "sink": 128, "window": 4096, "modes": "11111111",
         "new": "16384,777,6001,1500,300,4500,2160,1146", "past": "0,0,0,0,0,0,0,0"},
        # a chunk of each of four prompts, starting where the last chunk ended (chunks are whole blocks but for the last)
        {"name": "store_chunks", "op": "store", "fmt": "int8", "hq": 28, "hkv": 4, "sink": 128, "window": 4096, "modes": "1111",
         "new": "2048,2047,1000,4095", "past": "4096,2048,0,2064"},
        # one decode step's tokens of a batch: some of them complete a block, most do not
        {"name": "store_tokens", "op": "store", "fmt": "e4m3", **llama, "sink": 128, "window": 4096, "modes": "1" * 32,
         "new": _text([1] * 32), "past": _text([(37 * i * i + 11 * i) % 2000 for i in range(31)] + [15])},
        # a short chat, batch 1: latency of one launch
        {"name": "decode_short", "op": "decode", "fmt": "int8", "hq": 8, "hkv": 2, "sink": 64, "window": 256, "modes": "1", "ctx": "333"},
        # a large batch of short contexts: many small pieces of work
        {"name": "decode_wide", "op": "decode", "fmt": "e4m3", **llama, "sink": 128, "window": 2048, "modes": "10" * 32,
         "ctx": _text([100 + (397 * i * i + 61 * i) % 3900 for i in range(64)])},
        # a single long context (group of 7), dense
        {"name": "decode_long", "op": "decode", "fmt": "e4m3", "hq": 28, "hkv": 4, "sink": 128, "window": 4096, "modes": "1", "ctx": "131071"},
        # batched long-context decode, half of the requests sparse in this layer
        {"name": "decode_batch", "op": "decode", "fmt": "e4m3", **llama, "sink": 128, "window": 4096, "modes": "11010010",
         "ctx": _text([65536 + 7 * i for i in range(8)])},
        # ragged batch with mixed routing, the other 8-bit type
        {"name": "decode_ragged", "op": "decode", "fmt": "int8", **llama, "sink": 128, "window": 4096, "modes": "1011010110111001",
         "ctx": "4096,131072,20011,5003,64000,9999,30007,12288,7000,90017,17000,4444,50021,26000,8191,110000"},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    hq, hkv = rng.choice([(32, 8), (28, 4), (8, 2), (8, 8), (16, 1)])
    sink, window = rng.choice([(128, 4096), (128, 2048), (64, 256), (0, 500), (5, 33)])
    op = rng.choice(["prefill", "store", "decode", "decode"])
    case = {"op": op, "hq": hq, "hkv": hkv, "sink": sink, "window": window}
    if op == "decode":
        b = _spread(rng, 1, 64)
        most = min(131072, 560000 // b)
        return {**case, "fmt": rng.choice(["e4m3", "int8"]), "modes": "".join(rng.choice("01") for _ in range(b)),
                "ctx": _text(_spread(rng, 1, most) for _ in range(b))}
    b = _spread(rng, 1, 32)
    room = 32768 if op == "store" else 20000        # rows in all
    new, past = [], []
    for _ in range(b):
        n = min(room, _spread(rng, 1, 9000)) if rng.random() < 0.95 else 0
        p = 0 if rng.random() < 0.5 else _spread(rng, 1, 4096)
        if op == "store" and p % BLOCK:     # tokens that join a begun block, or a chunk from the next block on
            n, p = (min(n, BLOCK - p % BLOCK), p) if rng.random() < 0.5 else (n, p - p % BLOCK)
        room -= n
        new.append(n)
        past.append(p)
    if sum(new) == 0:
        new[0] = 1
    if op == "store":       # every position of a dense request stays readable
        return {**case, "fmt": rng.choice(["e4m3", "int8"]), "modes": "1" * b, "new": _text(new), "past": _text(past)}
    return {**case, "modes": "".join(rng.choice("01") for _ in range(b)), "new": _text(new), "past": _text(past)}


# ---- inputs -----------------------------------------------------------------------------------------------------

def _values(gen, rows, heads, spread):
    """Rows of a projection: unit noise whose channels differ in size (as those of keys do), a few of them large."""
    size = torch.exp(spread * torch.randn(heads, D, generator=gen, device=DEV))
    x = torch.empty(rows, heads, D, dtype=torch.bfloat16, device=DEV).normal_(generator=gen)
    return x.mul_(size.to(torch.bfloat16))


def _kept(ctx, fa, sink, window):
    """Positions that a decode step at length ctx may need of a request: all, or sink and window."""
    return ctx if fa or ctx <= sink + window else sink + window


def _plan(case, modes, max_context, compact):
    """The plan a program keeps for a layer: configuration, workspace, routing decision."""
    from paper_2604_07394_b200 import flux
    plan = flux.Plan(flux.make_config(1, case["hq"], case["hkv"], case["sink"], case["window"], len(modes), max_context,
                                      kv_layout=flux.FLUX_KV_COMPACT_SA if compact else flux.FLUX_KV_FULL), DEV)
    plan.flux_router_apply(mask=np.array([[int(m)] for m in modes], dtype=np.uint8))
    return flux, plan


def _fmt(flux, case):
    return flux.FLUX_KVQ_E4M3 if case["fmt"] == "e4m3" else flux.FLUX_KVQ_INT8


def _caches(flux, plan, modes, lens, compact):
    """Cache buffers of every request and the device tables of their addresses."""
    sizes = [flux.flux_kvq_cache_size(plan.cfg, compact and m == "0", n) for m, n in zip(modes, lens)]
    k = [torch.empty(s, dtype=torch.uint8, device=DEV) for s in sizes]
    v = [torch.empty(s, dtype=torch.uint8, device=DEV) for s in sizes]
    return k, v, flux.pointer_table(k, DEV), flux.pointer_table(v, DEV)


def _dev(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _sum(values):
    return [0] + list(np.cumsum(values))


def _inputs(case, seed):
    """What the seed alone makes: the bf16 tensors before any cache is filled, and the lengths."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed) * 7919 + 13)
    hq, hkv = case["hq"], case["hkv"]
    if case["op"] == "decode":
        ctx = _ints(case["ctx"])
        return {"ctx": ctx, "q": _values(gen, len(ctx), hq, 0.2),
                "k": _values(gen, sum(ctx), hkv, 0.5), "v": _values(gen, sum(ctx), hkv, 0.3)}
    new, past = _ints(case["new"]), _ints(case["past"])
    if case["op"] == "prefill":
        keys = [n + p if n else 0 for n, p in zip(new, past)]
        return {"new": new, "keys": keys, "q": _values(gen, sum(new), hq, 0.2),
                "k": _values(gen, sum(keys), hkv, 0.5), "v": _values(gen, sum(keys), hkv, 0.3)}
    head = [p % BLOCK if n else 0 for n, p in zip(new, past)]      # rows of the first block that are there already
    return {"new": new, "past": past, "head": head,
            "k": _values(gen, sum(new), hkv, 0.5), "v": _values(gen, sum(new), hkv, 0.3),
            "k0": _values(gen, sum(head), hkv, 0.5), "v0": _values(gen, sum(head), hkv, 0.3)}


def _blocks(new, head):
    """Rows of every block that the new rows touch, as indices into cat(earlier rows, new rows): (index [blocks][16],
    valid [blocks][16])."""
    at0, at1 = 0, sum(head)
    idx = []
    for n, h in zip(new, head):
        rows = list(range(at0, at0 + h)) + list(range(at1, at1 + n))
        at0, at1 = at0 + h, at1 + n
        idx += rows + [-1] * (-len(rows) % BLOCK)
    idx = torch.tensor(idx, device=DEV).reshape(-1, BLOCK)
    return idx.clamp(min=0), idx >= 0


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    modes = case["modes"]
    if case["op"] == "prefill":
        s["q_rows"], s["k_rows"] = np.array(_sum(s["new"]), dtype=np.int32), np.array(_sum(s["keys"]), dtype=np.int32)
        if own:
            s["flux"], s["plan"] = _plan(case, modes, max(s["keys"]), False)
    elif case["op"] == "store":
        s["index"], s["valid"] = _blocks(s["new"], s["head"])
        if own:
            ends = [n + p for n, p in zip(s["new"], s["past"])]
            s["flux"], s["plan"] = _plan(case, modes, max(ends), False)
            s["k_caches"], s["v_caches"], s["kt"], s["vt"] = _caches(s["flux"], s["plan"], modes, ends, False)
            s["rows"], s["pos"], s["ctx"] = _dev(_sum(s["new"])), _dev(s["past"]), _dev(ends)
            # what is read back: the touched blocks whole, so from the start of the first one
            s["out_rows"] = _dev(_sum([n + h for n, h in zip(s["new"], s["head"])]))
            s["out_pos"] = _dev([p - h for p, h in zip(s["past"], s["head"])])
            s["plan"].flux_kvq_store(0, _fmt(s["flux"], case), s["k0"], s["v0"], _dev(_sum(s["head"])), s["out_pos"], s["kt"], s["vt"])
    else:
        ctx = s["ctx"]
        k, v = s.pop("k"), s.pop("v")
        if own:
            s["flux"], s["plan"] = _plan(case, modes, max(ctx), True)
            s["k_caches"], s["v_caches"], s["kt"], s["vt"] = _caches(s["flux"], s["plan"], modes, ctx, True)
            s["ctx_dev"] = _dev(ctx)
            s["plan"].flux_kvq_store(0, _fmt(s["flux"], case), k, v, _dev(_sum(ctx)), _dev([0] * len(ctx)), s["kt"], s["vt"])
        else:
            s["cache"] = [[_held(x, case["fmt"]) for x in (k[a:b], v[a:b])] for a, b in zip(_sum(ctx), _sum(ctx)[1:])]
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------

def _scales(amax, fmt):
    """Scale of a block from its largest magnitude.  e4m3: the smallest power of two that brings it to 448 or below;
    int8: amax / 127.  A block of zeros has 1; neither goes below 2^-100."""
    if fmt == "e4m3":
        m, e = torch.frexp(amax)
        s = torch.ldexp(torch.ones_like(amax), torch.where(m <= 0.875, e - 9, e - 8))
    else:
        s = amax / 127.0
    return torch.where(amax == 0, torch.ones_like(s), s.clamp(min=2.0 ** -100))


def _codes(x, s, fmt):
    """x [blocks][16][heads][D] in 8 bits under the scales s [blocks][1][heads][1]; the int8 quotient in 64 bits, since it is rounded."""
    if fmt == "e4m3":
        return (x / s).to(torch.float8_e4m3fn)
    return torch.round(x.double() / s.double()).clamp(-127, 127).to(torch.int8)


def _held(x, fmt):
    """A cache's parts: codes and scales of the complete blocks, bf16 rows of the last one."""
    full = x.shape[0] // BLOCK * BLOCK
    b = x[:full].float().reshape(-1, BLOCK, *x.shape[1:])
    s = _scales(b.abs().amax((1, 3), keepdim=True), fmt)
    return _codes(b, s, fmt), s, x[full:]


def _stands_for(held):
    codes, s, tail = held
    return torch.cat([(codes.float() * s).reshape(-1, *tail.shape[1:]), tail.float()])


def _attend(q, k, v, first, keys, fa, sink, window):
    """Rows q [n][hq][D] at positions first.. over k, v [keys][hkv][D] in 32 bits; a row sees the positions up to its own,
    a sparse request's row only the sink and its window."""
    n, hq = q.shape[:2]
    hkv = k.shape[1]
    at = torch.arange(first, first + n, device=q.device)[:, None]
    j = torch.arange(keys, device=q.device)[None, :]
    keep = j <= at
    if not fa:
        keep = keep & ((j < sink) | (j > at - window))
    g = q.reshape(n, hkv, hq // hkv, D).permute(1, 2, 0, 3).reshape(hkv, -1, D)
    s = (g @ k.permute(1, 2, 0)).reshape(hkv, -1, n, keys) / math.sqrt(D)
    s = torch.where(keep, s, torch.full_like(s, -math.inf))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = (p.reshape(hkv, -1, keys) @ v.permute(1, 0, 2)).reshape(hkv, -1, n, D) / p.sum(-1)[..., None]
    return o.permute(2, 0, 1, 3).reshape(n, hq, D)


def _plain_prefill(s):
    case = s["case"]
    out = torch.empty_like(s["q"])
    for b, m in enumerate(case["modes"]):       # requests differ in length; a dense score matrix of all would not fit
        q0, q1, k0, k1 = s["q_rows"][b], s["q_rows"][b + 1], s["k_rows"][b], s["k_rows"][b + 1]
        k, v = s["k"][k0:k1].float(), s["v"][k0:k1].float()
        for r in range(q0, q1, 2048):           # nor one of a long prompt's rows
            e = min(r + 2048, q1)
            last = k1 - k0 - (q1 - e)           # keys up to the last row's own
            out[r:e] = _attend(s["q"][r:e].float(), k[:last], v[:last], last - (e - r), last, m == "1", case["sink"], case["window"]).to(torch.bfloat16)
    return out


def _plain_store(s):
    fmt, found = s["case"]["fmt"], []
    for old, new in ((s["k0"], s["k"]), (s["v0"], s["v"])):
        x = torch.cat([old, new]).float()[s["index"]]
        sc = _scales(x.abs().amax((1, 3), keepdim=True), fmt)
        y = _codes(x, sc, fmt).float() * sc
        y = torch.where(s["valid"].all(1)[:, None, None, None], y, x)      # an incomplete block stays as it is
        found.append(y.to(torch.bfloat16)[s["valid"]])
    return found


def _plain_decode(s):
    case = s["case"]
    out = torch.empty_like(s["q"])
    for b, (n, m) in enumerate(zip(s["ctx"], case["modes"])):       # requests differ in length
        k, v = (_stands_for(h) for h in s["cache"][b])
        out[b] = _attend(s["q"][b:b + 1].float(), k, v, n - 1, n, m == "1", case["sink"], case["window"])[0].to(torch.bfloat16)
    return out


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"prefill": _plain_prefill, "store": _plain_store, "decode": _plain_decode}[op](s)
    plan = s["plan"]
    if op == "prefill":
        return plan.flux_attn_prefill_packed(0, s["q"], s["k"], s["v"], s["q_rows"], s["k_rows"])
    fmt = _fmt(s["flux"], s["case"])
    if op == "store":
        plan.flux_kvq_store(0, fmt, s["k"], s["v"], s["rows"], s["pos"], s["kt"], s["vt"])
        return plan.flux_kvq_load(0, fmt, s["kt"], s["vt"], s["ctx"], s["out_rows"], s["out_pos"], sum(s["new"]) + sum(s["head"]))
    return plan.flux_attn_decode_kvq(0, len(s["ctx"]), fmt, s["q"], s["kt"], s["vt"], s["ctx_dev"])


# ---- work and exact values --------------------------------------------------------------------------------------

def work(case):
    hq, hkv, sink, window = case["hq"], case["hkv"], case["sink"], case["window"]
    modes = case["modes"]
    if case["op"] == "decode":
        ctx = _ints(case["ctx"])
        rows = tail = 0
        for n, m in zip(ctx, modes):
            t = min(n % BLOCK, _kept(n, m == "1", sink, window))
            tail += t
            rows += _kept(n, m == "1", sink, window) - t
        return {"bytes": 2 * hkv * (rows * D + rows // BLOCK * 4 + tail * 2 * D) + 2 * len(ctx) * hq * D * 2,
                "flops": 4 * hq * D * (rows + tail)}
    new, past = _ints(case["new"]), _ints(case["past"])
    if case["op"] == "store":       # rows in, 8 bits and scales out and in again, values out
        head = [p % BLOCK if n else 0 for n, p in zip(new, past)]
        full = sum((n + h) // BLOCK * BLOCK for n, h in zip(new, head))
        touched = sum(new) + sum(head)
        row = hkv * D * 2
        held = full * row // 2 + full // BLOCK * hkv * 4 + (touched - full) * row
        return {"bytes": 2 * (row * touched + 2 * held + row * touched), "flops": 0}
    rows = pairs = keys = 0
    for n, p, m in zip(new, past, modes):
        if not n:
            continue
        i = np.arange(p, p + n, dtype=np.int64) + 1
        seen = i if m == "1" else np.minimum(i, sink + window)
        rows += n
        pairs += int(seen.sum())
        first = 0 if m == "1" else max(0, p + 1 - window)       # keys before the first row's window, but for the sink, are not needed
        keys += n + p - max(0, first - sink)
    return {"bytes": 2 * D * (2 * hq * rows + 2 * hkv * keys), "flops": 4 * hq * D * pairs}


def _exact_block(x, fmt):
    """Values that the 8-bit codes of a block x [16][heads][D] (64 bits) stand for, by the definition of the two types."""
    top = x.abs().amax((0, 2), keepdim=True)
    if fmt == "int8":
        s = torch.clamp((top / 127).float().double(), min=2.0 ** -100)
        s = torch.where(top == 0, torch.ones_like(s), s)
        return torch.clamp(torch.round(x / s), -127, 127) * s
    s = torch.exp2(torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 448) - 1e-12)).clamp(min=2.0 ** -100)
    s = torch.where(top == 0, torch.ones_like(s), s)
    y = x / s
    # three fraction bits, smallest normal exponent -6
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * s


def _exact_values(x, fmt):
    """Each complete block of x [n][heads][D] as its codes stand for it, the rest as it is."""
    x = x.double()
    full = x.shape[0] // BLOCK * BLOCK
    if full == 0:
        return x
    blocks = x[:full].reshape(-1, BLOCK, *x.shape[1:]).transpose(0, 1).reshape(BLOCK, -1, D)     # blocks beside heads
    y = _exact_block(blocks, fmt).reshape(BLOCK, full // BLOCK, -1, D).transpose(0, 1).reshape(full, -1, D)
    return torch.cat([y, x[full:]])


def _exact_rows(q, k, v, at, fa, sink, window):
    """softmax(q K^T / sqrt(D)) V in 64 bits for rows at the positions `at`, one KV head after another."""
    n, hq = q.shape[:2]
    hkv, keys = k.shape[1], k.shape[0]
    j = torch.arange(keys, device=DEV)
    hidden = j[None, :] > at[:, None]
    if not fa:
        hidden |= (j[None, :] >= sink) & (at[:, None] - j[None, :] >= window)
    out = torch.empty(n, hq, D, dtype=torch.float64, device=DEV)
    for h in range(hq):
        kv = h // (hq // hkv)
        s = (q[:, h].double() @ k[:, kv].double().T) * (1.0 / math.sqrt(D))
        s.masked_fill_(hidden, -math.inf)
        s -= s.max(1, keepdim=True).values
        s.exp_()
        out[:, h] = (s @ v[:, kv].double()) / s.sum(1, keepdim=True)
    return out


def exact(case, seed):
    x = _inputs(case, seed)
    sink, window, fmt = case["sink"], case["window"], case.get("fmt")
    if case["op"] == "store":
        found = []
        for old, new in ((x["k0"], x["k"]), (x["v0"], x["v"])):
            a = b = 0
            parts = []
            for n, h in zip(x["new"], x["head"]):
                parts.append(_exact_values(torch.cat([old[a:a + h], new[b:b + n]]), fmt))
                a, b = a + h, b + n
            found.append(torch.cat(parts))
        return found
    out = torch.empty(x["q"].shape, dtype=torch.float64, device=DEV)
    a = b = 0
    if case["op"] == "decode":
        for i, (n, m) in enumerate(zip(x["ctx"], case["modes"])):
            k, v = (_exact_values(t[a:a + n], fmt) for t in (x["k"], x["v"]))
            out[i:i + 1] = _exact_rows(x["q"][i:i + 1], k, v, torch.tensor([n - 1], device=DEV), m == "1", sink, window)
            a += n
        return out
    for n, keys, m in zip(x["new"], x["keys"], case["modes"]):
        k, v = x["k"][b:b + keys], x["v"][b:b + keys]
        for r in range(0, n, 4096):
            e = min(n, r + 4096)
            at = torch.arange(keys - n + r, keys - n + e, device=DEV)
            last = keys - n + e
            out[a + r:a + e] = _exact_rows(x["q"][a + r:a + e], k[:last], v[:last], at, m == "1", sink, window)
        a, b = a + n, b + keys
    return out
