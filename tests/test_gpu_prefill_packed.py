"""GPU parity of the packed prefill (flux_attn_prefill_packed): against the fp64 oracle row by row, and bit for bit against
flux_attn_prefill of each request alone (the same tiles in the same order).  The oracle comparison is the one rule of
tests/_util.py, which the single-request prefill is held to."""
import numpy as np
import pytest
import torch

import oracle
from tests._util import bits, compare

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def flux():
    from paper_2604_07394_b200 import build, flux as f
    build.build()
    f.load()
    return f


def _cum(x, first=0):
    return np.array([first] + (first + np.cumsum(x)).tolist(), dtype=np.int32)


def _plan(flux, Hq, Hkv, S, W, modes, max_ctx):
    plan = flux.Plan(flux.make_config(1, Hq, Hkv, S, W, len(modes), max_ctx), DEV)
    plan.flux_router_apply(mask=np.array([[m] for m in modes], dtype=np.uint8))
    return plan


def _rows(n, heads, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(n, heads, 128, generator=g, device=DEV).to(torch.bfloat16)


def _check(flux, Hq, Hkv, S, W, modes, new, past, seed=1, against_oracle=True):
    keys = [n + p for n, p in zip(new, past)]
    plan = _plan(flux, Hq, Hkv, S, W, modes, max(max(keys), 1))
    q, k, v = _rows(sum(new), Hq, seed), _rows(sum(keys), Hkv, seed + 1), _rows(sum(keys), Hkv, seed + 2)
    qr, kr = _cum(new), _cum(keys)
    out = plan.flux_attn_prefill_packed(0, q, k, v, qr, kr)
    rec = plan.flux_debug_dispatch(len(modes))
    for b, m in enumerate(modes):
        assert rec[b, 0] == (m if new[b] else -1) and rec[b, 2] == b
        if not new[b]:
            continue
        kb, vb, qb = k[kr[b]:kr[b + 1]].contiguous(), v[kr[b]:kr[b + 1]].contiguous(), q[qr[b]:qr[b + 1]].contiguous()
        single = plan.flux_attn_prefill(0, b, qb, kb, vb, past[b])
        assert torch.equal(single, out[qr[b]:qr[b + 1]]), "request %d" % b
        if against_oracle:
            ref = oracle.prefill(m, bits(qb), bits(kb), bits(vb), past[b], S, W, 1 / np.sqrt(128))
            compare(out[qr[b]:qr[b + 1]], ref, "request %d" % b)
        assert rec[b, 3] == keys[b]
        n = keys[b]
        assert rec[b].tolist()[4:] == ([0, S, n - W, n] if m == 0 and n > S + W else [0, n, 0, 0])
    assert plan.flux_plan_status() == 0
    return plan


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 1), (8, 2), (7, 1), (28, 4), (8, 8), (16, 1), (3, 3)])
def test_head_layouts_and_lengths(flux, Hq, Hkv):
    new = [1, 0, 127, 128, 129, 300, 2, 257, 0, 513, 64, 255]
    modes = [1, 0, 0, 1, 0, 1, 0, 0, 1, 0, 1, 1]
    _check(flux, Hq, Hkv, 20, 70, modes, new, [0] * len(new), seed=Hq)


@pytest.mark.parametrize("S,W", [(0, 1), (5, 33), (64, 256), (130, 300)])
def test_chunks_behind_earlier_keys(flux, S, W):
    new = [1, 100, 0, 200, 129, 384, 1, 17]
    past = [1, 0, 50, 130, 1000, 77, 640, 3]
    for modes in ([0] * 8, [1, 0] * 4):
        _check(flux, 8, 2, S, W, modes, new, past, seed=S)


def _tolerance(ref, q, k, v, past, fa, S, W):
    """What an element may be off by whatever the weights p_j (tests/_util.py's rule is for the flat weights of N(0, 1) keys):
    2^-8 |ref| (bf16 output) + 2^-8 A (weights rounded to bf16, A = sum_j p_j |v_j|) + 2 D A (weights off by a factor 1 + D in
    numerator and row sum: D = 2^-20 for ex2, fp32 sums and rescaling, + the error of a score, 2^-16 of the largest sum_d |q_d k_jd|
    for 128 fp32 additions of exact products in any order, rounded or cut off)."""
    n, hq = q.shape[:2]
    G = hq // k.shape[1]
    qd, kd, vd = q.double(), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    at, j = torch.arange(past, past + n, device=DEV)[:, None], torch.arange(k.shape[0], device=DEV)[None, :]
    keep = (j <= at) if fa else (j <= at) & ((j < S) | (j > at - W))
    s = torch.einsum("nhd,jhd->hnj", qd, kd) / np.sqrt(128)
    p = torch.softmax(s.masked_fill(~keep, -np.inf), -1)
    A = torch.einsum("hnj,jhd->nhd", p, vd.abs())
    mag = (torch.einsum("nhd,jhd->hnj", qd.abs(), kd.abs()) / np.sqrt(128)).masked_fill(~keep, 0).amax(-1).T[..., None]
    return (2.0 ** -8 * (torch.from_numpy(ref).to(DEV).abs() + A) + 2 * (2.0 ** -20 + 2.0 ** -16 * mag) * A).cpu().numpy()


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (7, 1), (3, 3), (16, 1)])
@pytest.mark.parametrize("new,past", [([1], [5000]), ([5, 1, 0, 130], [4000, 3001, 10, 2500]), ([300], [4800]), ([1, 129, 40, 2], [6000, 100, 0, 1536])])
def test_few_rows_over_many_keys(flux, Hq, Hkv, new, past):
    """Items cut along the keys and added up: against the oracle, and the same bits each time."""
    S, W = 130, 1000
    keys = [n + p if n else 0 for n, p in zip(new, past)]
    q, k, v = _rows(sum(new), Hq, Hq), _rows(sum(keys), Hkv, 8), _rows(sum(keys), Hkv, 9)
    k[::37] *= 3                               # some scores stand out, so that the parts' maxima differ
    qr, kr = _cum(new), _cum(keys)
    for modes in ([1] * len(new), [0] * len(new)):
        plan = _plan(flux, Hq, Hkv, S, W, modes, 7000)
        out = plan.flux_attn_prefill_packed(0, q, k, v, qr, kr)
        for _ in range(4):
            assert torch.equal(out, plan.flux_attn_prefill_packed(0, q, k, v, qr, kr))
        for b, m in enumerate(modes):
            if new[b]:
                x = q[qr[b]:qr[b + 1]], k[kr[b]:kr[b + 1]], v[kr[b]:kr[b + 1]]
                ref = np.asarray(oracle.prefill(m, *[bits(t) for t in x], past[b], S, W, 1 / np.sqrt(128))).reshape(x[0].shape)
                over = np.abs(out[qr[b]:qr[b + 1]].double().cpu().numpy() - ref) / _tolerance(ref, *x, past[b], m == 1, S, W)
                assert over.max() <= 1, "request %d: %.2f of the tolerance" % (b, over.max())
        rec = plan.flux_debug_dispatch(len(new))
        assert rec[:, 0].tolist() == [m if n else -1 for m, n in zip(modes, new)] and rec[:, 3].tolist() == keys
        assert plan.flux_plan_status() == 0


def test_one_request_of_each_length(flux):
    for n in (1, 128, 130):
        _check(flux, 8, 2, 4, 8, [0], [n], [0], seed=n)


def test_more_requests_than_one_launch_takes(flux):
    rng = np.random.default_rng(4)
    B = 300
    new = [int(x) for x in rng.integers(0, 40, B)]
    new[7], new[290] = 700, 400
    past = [int(x) for x in rng.integers(0, 30, B)]
    plan = _check(flux, 4, 2, 8, 16, [int(x) for x in rng.integers(0, 2, B)], new, past, against_oracle=False)
    before = plan.flux_launch_count()
    x, y = _rows(sum(new), 4, 3), _rows(sum(new), 2, 5)
    plan.flux_attn_prefill_packed(0, x, y, y, _cum(new))
    assert plan.flux_launch_count() - before == 5          # 64 requests each


def test_many_items_per_block_and_repeats(flux):
    """Enough work that every block draws many items; the same call again gives the same bits (the counter is back at zero)."""
    new = [5000, 3000, 100, 2500, 1, 700]
    plan = _plan(flux, 14, 2, 128, 512, [1, 0, 1, 0, 1, 0], 5000)
    q, k, v = _rows(sum(new), 14, 1), _rows(sum(new), 2, 2), _rows(sum(new), 2, 3)
    qr = _cum(new)
    out = plan.flux_attn_prefill_packed(0, q, k, v, qr)
    for _ in range(5):
        assert torch.equal(out, plan.flux_attn_prefill_packed(0, q, k, v, qr))
    for b in range(6):
        single = plan.flux_attn_prefill(0, b, q[qr[b]:qr[b + 1]].contiguous(), k[qr[b]:qr[b + 1]].contiguous(), v[qr[b]:qr[b + 1]].contiguous(), 0)
        assert torch.equal(single, out[qr[b]:qr[b + 1]])
    assert plan.flux_plan_status() == 0


def test_strided_rows_and_rows_left_alone(flux):
    """q, k, v as slices of one fused projection output; rows before, behind and between the requests hold NaN and infinities."""
    Hq, Hkv, new = 8, 2, [150, 33, 200]
    plan = _plan(flux, Hq, Hkv, 16, 64, [1, 0, 1], 300)
    fused = _rows(420, Hq + 2 * Hkv, 3)
    rows = _cum(new, 10)                     # rows 0..9 and from 393 on belong to nobody
    fused[:10] = float("nan")
    fused[393:] = float("inf")
    fused[393::2] = float("nan")
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    out = torch.full((420, Hq, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    plan.flux_attn_prefill_packed(0, q, k, v, rows, out=out)
    assert bool((out[:10] == 7).all()) and bool((out[393:] == 7).all())
    for b in range(3):
        a, e = rows[b], rows[b + 1]
        single = plan.flux_attn_prefill(0, b, q[a:e].contiguous(), k[a:e].contiguous(), v[a:e].contiguous(), 0)
        assert torch.equal(single, out[a:e]), b
    assert plan.flux_plan_status() == 0


def test_requests_do_not_see_each_others_values(flux):
    """NaN and infinities in one request (keys, values, queries) leave the others' bits as they were."""
    Hq, Hkv, new = 6, 2, [130, 100, 129, 5, 260, 127]
    plan = _plan(flux, Hq, Hkv, 16, 64, [1, 0, 1, 0, 1, 0], 300)
    q, k, v = _rows(sum(new), Hq, 1), _rows(sum(new), Hkv, 2), _rows(sum(new), Hkv, 3)
    rows = _cum(new)
    want = plan.flux_attn_prefill_packed(0, q, k, v, rows)
    for bad in (1, 3, 4):
        a, e = rows[bad], rows[bad + 1]
        for val in (float("nan"), float("inf"), -float("inf")):
            q2, k2, v2 = q.clone(), k.clone(), v.clone()
            for x in (q2, k2, v2):
                x[a:e] = val
            out = plan.flux_attn_prefill_packed(0, q2, k2, v2, rows)
            assert torch.equal(out[:a], want[:a]) and torch.equal(out[e:], want[e:])
    assert plan.flux_plan_status() == 0


def test_touched_positions(flux):
    plan = _plan(flux, 4, 2, 16, 64, [1, 0], 700)
    new, past = [200, 129], [0, 500]
    keys = [200, 629]
    q, k, v = _rows(329, 4, 1), _rows(829, 2, 2), _rows(829, 2, 3)
    bitmap = torch.zeros((2, 22), dtype=torch.int32, device=DEV)
    plan.flux_debug_touched(bitmap)
    plan.flux_attn_prefill_packed(0, q, k, v, _cum(new), _cum(keys))
    plan.flux_debug_touched(None)
    words = bitmap.cpu().numpy().view(np.uint32)
    seen = [[p for p in range(704) if words[b, p // 32] >> (p % 32) & 1] for b in range(2)]
    assert seen[0] == list(range(200))
    assert seen[1] == list(range(128)) + list(range(384, 629))      # the sink's tile, and from the tile of 500 - 64 + 1 on


def test_prefill_store_load_chunk_decode_chain(flux):
    """The calls as a server makes them: packed prompts, 8-bit caches, a second chunk over what the caches hold, decode steps."""
    from oracle import kvq
    Hq, Hkv, S, W, modes = 8, 2, 16, 64, [1, 0, 1]
    plan = _plan(flux, Hq, Hkv, S, W, modes, 600)
    fmt = flux.FLUX_KVQ_INT8
    first, second = [300, 129, 64], [100, 0, 200]
    q, k, v = _rows(493, Hq, 1), _rows(493, Hkv, 2), _rows(493, Hkv, 3)
    r1 = _cum(first)
    out1 = plan.flux_attn_prefill_packed(0, q, k, v, r1)
    bufs = [[torch.empty(flux.flux_kvq_cache_size(plan.cfg, False, 600), dtype=torch.uint8, device=DEV) for _ in modes] for _ in "kv"]
    kt, vt = (flux.pointer_table(b, DEV) for b in bufs)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    plan.flux_kvq_store(0, fmt, k, v, dev(r1.tolist()), dev([0, 0, 0]), kt, vt)
    # second chunk: earlier positions as the caches hold them, the chunk's own rows behind them
    k2, v2 = _rows(300, Hkv, 5), _rows(300, Hkv, 6)
    q2 = _rows(300, Hq, 7)
    old = [f if s else 0 for f, s in zip(first, second)]
    keys = [o + s for o, s in zip(old, second)]
    kr, orow, r2 = _cum(keys), _cum(old), _cum(second)
    ko, vo = plan.flux_kvq_load(0, fmt, kt, vt, dev(first), dev(orow.tolist()), dev([0, 0, 0]), int(orow[-1]))
    kc = torch.cat([torch.cat([ko[orow[b]:orow[b + 1]], k2[r2[b]:r2[b + 1]]]) for b in range(3)])
    vc = torch.cat([torch.cat([vo[orow[b]:orow[b + 1]], v2[r2[b]:r2[b + 1]]]) for b in range(3)])
    out2 = plan.flux_attn_prefill_packed(0, q2, kc, vc, r2, kr)
    plan.flux_kvq_store(0, fmt, k2, v2, dev(r2.tolist()), dev(first), kt, vt)
    hist = [[torch.cat([x[r1[b]:r1[b + 1]], y[r2[b]:r2[b + 1]]]) for b in range(3)] for x, y in ((k, k2), (v, v2))]
    for b in range(3):
        a, e = r1[b], r1[b + 1]
        compare(out1[a:e], oracle.prefill(modes[b], bits(q[a:e]), bits(k[a:e]), bits(v[a:e]), 0, S, W, 1 / np.sqrt(128)), "first chunk")
        a, e = r2[b], r2[b + 1]
        if e > a:
            kk, vv = kc[kr[b]:kr[b + 1]], vc[kr[b]:kr[b + 1]]
            compare(out2[a:e], oracle.prefill(modes[b], bits(q2[a:e]), bits(kk), bits(vv), first[b], S, W, 1 / np.sqrt(128)), "second chunk")
    for step in range(20):
        kn, vn, qd = _rows(3, Hkv, 100 + step), _rows(3, Hkv, 200 + step), _rows(3, Hq, 300 + step)
        hist = [[torch.cat([h[b], x[b:b + 1]]) for b in range(3)] for h, x in zip(hist, (kn, vn))]
        ctx = [len(h) for h in hist[0]]
        out = plan.flux_attn_decode_step_kvq(0, 3, fmt, qd, kn, vn, kt, vt, dev(ctx))
        for b in range(3):
            keep = kvq.kept(ctx[b], modes[b] == 1, S, W)
            vals = [kvq.cache_values(h[b].double().cpu().numpy(), "int8")[keep] for h in hist]
            ref = kvq.attend(qd[b].double().cpu().numpy(), vals[0], vals[1], 1 / np.sqrt(128))[0]
            compare(out[b], ref, "step %d" % step)
    assert plan.flux_plan_status() == 0


def test_replays_follow_the_inputs_and_the_routing(flux):
    """A captured call (some items cut along the keys, some not) replayed over other rows and after other routing decisions."""
    new, past = [3, 200, 1, 700], [5000, 900, 2600, 0]
    keys = [n + p for n, p in zip(new, past)]
    qr, kr = _cum(new), _cum(keys)
    plan, other = (_plan(flux, 8, 2, 64, 256, [1, 1, 1, 1], max(keys)) for _ in range(2))
    q, k, v = _rows(sum(new), 8, 1), _rows(sum(keys), 2, 2), _rows(sum(keys), 2, 3)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        plan.flux_attn_prefill_packed(0, q, k, v, qr, kr, out)
    for i, modes in enumerate(([1, 0, 1, 0], [0, 0, 0, 0], [0, 1, 1, 1], [1, 1, 0, 0], [1, 1, 1, 1])):
        mask = np.array([[m] for m in modes], dtype=np.uint8)
        plan.flux_router_apply(mask=mask, mask_out=plan.mask)      # the captured launch reads the decision from there
        other.flux_router_apply(mask=mask)
        for t, heads in ((q, 8), (k, 2), (v, 2)):
            t.copy_(_rows(t.shape[0], heads, 10 + 3 * i + heads))
        g.replay()
        want = other.flux_attn_prefill_packed(0, q, k, v, qr, kr)
        assert bool(torch.equal(out, want)), modes
    assert plan.flux_plan_status() == 0 and other.flux_plan_status() == 0


def test_two_plans_on_two_streams_at_once(flux):
    """Each plan has its own workspace, so the calls of two plans may run at the same time: prompts with cut items beside stores and decodes."""
    new, past = [2, 300, 64], [4000, 0, 6000]
    keys = [n + p for n, p in zip(new, past)]
    qr, kr = _cum(new), _cum(keys)
    plan = _plan(flux, 8, 2, 64, 256, [1, 0, 1], max(keys))
    q, k, v = _rows(sum(new), 8, 1), _rows(sum(keys), 2, 2), _rows(sum(keys), 2, 3)
    want = plan.flux_attn_prefill_packed(0, q, k, v, qr, kr)
    fmt = flux.FLUX_KVQ_E4M3
    dec = _plan(flux, 8, 2, 64, 256, [1, 0, 1], max(keys))
    size = flux.flux_kvq_cache_size(dec.cfg, False, max(keys))
    bufs = [[torch.zeros(size, dtype=torch.uint8, device=DEV) for _ in keys] for _ in "kv"]
    kt, vt = (flux.pointer_table(b, DEV) for b in bufs)
    rows, zero, ctx = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (kr.tolist(), [0, 0, 0], keys))
    qd = _rows(3, 8, 5)
    dec.flux_kvq_store(0, fmt, k, v, rows, zero, kt, vt)
    want_d = dec.flux_attn_decode_kvq(0, 3, fmt, qd, kt, vt, ctx)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    outs, outs_d = [], []
    for _ in range(40):
        with torch.cuda.stream(one):
            outs.append(plan.flux_attn_prefill_packed(0, q, k, v, qr, kr))
        with torch.cuda.stream(two):
            dec.flux_kvq_store(0, fmt, k, v, rows, zero, kt, vt)
            outs_d.append(dec.flux_attn_decode_kvq(0, 3, fmt, qd, kt, vt, ctx))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in outs) and all(torch.equal(x, want_d) for x in outs_d)
    assert plan.flux_plan_status() == 0 and dec.flux_plan_status() == 0


def test_refusals(flux):
    plan = _plan(flux, 4, 2, 8, 16, [1, 0], 100)
    q, k = _rows(60, 4, 1), _rows(60, 2, 2)
    call = lambda qr, kr=None, **kw: plan.flux_attn_prefill_packed(kw.get("layer", 0), kw.get("q", q), kw.get("k", k), kw.get("v", k),  # noqa: E731
                                                                   qr, kr, kw.get("out"))
    for qr, kr, code in (([0, 10, 5], None, flux.FLUX_E_INVALID_ARG), ([-1, 10, 20], None, flux.FLUX_E_INVALID_ARG),
                         ([0, 30, 60], [0, 20, 50], flux.FLUX_E_INVALID_ARG), ([0, 1, 2, 3], None, flux.FLUX_E_CAPACITY)):
        with pytest.raises(flux.FluxError) as e:
            call(qr, kr)
        assert e.value.code == code
    big = _rows(300, 2, 2)
    with pytest.raises(flux.FluxError) as e:
        call([0, 10, 10], [0, 101, 101], k=big, v=big)
    assert e.value.code == flux.FLUX_E_CAPACITY
    with pytest.raises(flux.FluxError) as e:
        call([0, 10, 20], layer=1)
    assert e.value.code == flux.FLUX_E_INVALID_ARG
    odd = torch.zeros(60 * 4 * 128 + 8, dtype=torch.bfloat16, device=DEV)[4:4 + 60 * 4 * 128].view(60, 4, 128)     # 8 bytes off
    with pytest.raises(flux.FluxError) as e:
        call([0, 10, 20], q=odd)
    assert e.value.code == flux.FLUX_E_INVALID_ARG
    for kw in ({"q": q.float()}, {"q": _rows(60, 8, 1)[:, ::2]}, {"k": k[:10]}, {"out": q[:19]}, {"out": q.transpose(0, 1)}):
        with pytest.raises(ValueError):
            call([0, 10, 20], **kw)
    with pytest.raises(ValueError):
        call([0])
    assert call([0, 0, 0]).shape == q.shape and call([5, 5, 5]).shape == q.shape
    assert plan.flux_plan_status() == 0
