"""The paged calls at entries, counts and orders of calls that the parity tests leave out.  Without a stated tolerance what is compared here is exact: where
an entry of a head is not finite the others must have the bits that they have without it."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def flux():
    from paper_2604_07394_b200 import build, flux as f
    build.build()
    f.load()
    return f


def _dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _plan(flux, Hq, Hkv, S=4, W=8, modes=(1,), max_ctx=1 << 20):
    plan = flux.Plan(flux.make_config(1, Hq, Hkv, S, W, len(modes), max_ctx), DEV)
    plan.flux_router_apply(mask=np.array([[m] for m in modes], dtype=np.uint8))
    return plan


def _rows(seed, n, heads):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(n, heads, 128, generator=g, device=DEV).to(torch.bfloat16)


def _bits(x):
    return x.view(torch.int16)


def _inv_freq(rot):
    return 1e4 ** (-np.arange(0, rot, 2) / max(rot, 1))


# ---- channels that are not rotated -------------------------------------------------------------------------------------

def _spoiled(x, rot):
    """x with non-finite entries in channels from rot on, one of each kind in heads of their own and several in one; and where they are."""
    x = x.clone()
    n, heads = x.shape[:2]
    for i in range(n):
        for j, value in enumerate((INF, -INF, NAN)):
            x[i, (i + j) % heads, rot + (i * 7 + j * 13) % (128 - rot)] = value
    return x, ~torch.isfinite(x)


@pytest.mark.parametrize("n", [5, 2500])
@pytest.mark.parametrize("rot,pairs", [(64, False), (64, True), (96, False), (112, True), (16, False), (0, False), (0, True)])
def test_non_finite_entries_behind_the_rotated_channels(flux, rot, pairs, n):
    """Without a weight those channels pass as they are, so an infinity or a NaN in one of them is in that one alone: rows to rows, and stored,
    for few rows (dealt out by fours of heads) and many (whole rows)."""
    Hq, Hkv, page = 6, 3, 16
    plan = _plan(flux, Hq, Hkv)
    rope = flux.Rope(_inv_freq(rot), interleaved=pairs, device=DEV)
    q, k, v = (_rows(rot + z, n, h) for z, h in enumerate((Hq, Hkv, Hkv)))
    pos = _dev((np.arange(n) * 37) % 5000)
    (bq, at_q), (bk, at_k) = _spoiled(q, rot), _spoiled(k, rot)
    want, got = plan.flux_qk_norm_rope(rope, q, k, pos), plan.flux_qk_norm_rope(rope, bq, bk, pos)
    for x, y, bad, at in zip(want, got, (bq, bk), (at_q, at_k)):
        assert torch.equal(_bits(x)[~at], _bits(y)[~at])
        assert torch.equal(torch.isnan(y)[at], torch.isnan(bad)[at]) and torch.equal(y[torch.isinf(bad)], bad[torch.isinf(bad)])
    # a sample against the oracle, which leaves these channels alone
    some = [0, n // 2, n - 1]
    ref, mag = paged.turned(bk[some].double().cpu().numpy(), pos[some].tolist(), _inv_freq(rot), pairs=pairs)
    y, fine = got[1][some].double().cpu().numpy(), ~at_k[some].cpu().numpy()
    assert (np.abs(y[fine] - ref[fine]) <= 2.0 ** -8 * np.abs(ref[fine]) + 2.0 ** -17 * mag[fine]).all()
    assert np.array_equal(y[~fine], ref[~fine], equal_nan=True)
    # the same into pages
    cols = -(-n // page)
    pools = [torch.zeros(cols, page, Hkv, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    pages = flux.Pages(*pools, _dev(np.random.default_rng(n).permutation(cols)[None]))
    k_out = torch.empty_like(k)
    turned = plan.flux_paged_store(pages, bk, v, _dev([0, n]), _dev([0]), rope=rope, q=bq, k_out=k_out)
    straight = plan.flux_qk_norm_rope(rope, bq, bk, _dev(np.arange(n)))
    clean = plan.flux_qk_norm_rope(rope, q, k, _dev(np.arange(n)))
    for y, s, x, at in ((turned, straight[0], clean[0], at_q), (k_out, straight[1], clean[1], at_k)):
        assert torch.equal(_bits(y), _bits(s)) and torch.equal(_bits(y)[~at], _bits(x)[~at])
    lk, _ = plan.flux_paged_load(pages, _dev([n]), _dev([0, n]), _dev([0]), n)
    assert torch.equal(_bits(lk), _bits(k_out)) and plan.flux_plan_status() == 0


@pytest.mark.parametrize("rot,pairs", [(64, False), (64, True), (0, False)])
def test_a_step_stores_non_finite_entries_as_they_are(flux, rot, pairs):
    """The newest key's channels behind the rotated ones, through the step: the row in the page is the one that the store puts there, and heads
    whose key is finite have the outputs that they have without the entry."""
    Hq, Hkv, page, ctx = 8, 4, 16, [40, 100, 1]
    rope = flux.Rope(_inv_freq(rot), interleaved=pairs, device=DEV)
    plan = _plan(flux, Hq, Hkv, modes=(1, 0, 1), S=16, W=32)
    cols = 7
    table = _dev(np.arange(3 * cols).reshape(3, cols))
    q, k, v = (_rows(z, 3, h) for z, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    bad = k.clone()
    bad[0, 1, rot + 5], bad[1, 2, 127], bad[2, 3, rot] = NAN, INF, -INF
    found = []
    for key in (k, bad):
        pools = [_rows(9 + z, 3 * cols * page, Hkv).view(3 * cols, page, Hkv, 128) for z in range(2)]
        out = plan.flux_attn_decode_step_paged(0, 3, q, key, v, flux.Pages(*pools, table), _dev(ctx), rope=rope)
        found.append((out.view(3, Hkv, 2, 128), pools[0], pools[1]))
    slots = [(b * cols + (n - 1) // page, (n - 1) % page) for b, n in enumerate(ctx)]
    want = plan.flux_qk_norm_rope(rope, None, bad, _dev([n - 1 for n in ctx]))[1]
    for b, (p, r) in enumerate(slots):
        assert torch.equal(_bits(found[1][1][p, r]), _bits(want[b]))
        here, there = _bits(found[1][1][p, r]).clone(), _bits(found[0][1][p, r]).clone()
        fine = torch.isfinite(bad[b])
        assert torch.equal(here[fine], there[fine])
        heads = fine.all(-1)
        assert int(heads.sum()) == Hkv - 1 and torch.equal(found[1][0][b][heads], found[0][0][b][heads])
    assert torch.equal(found[0][2], found[1][2]) and plan.flux_plan_status() == 0


# ---- page calls with launch overlap ------------------------------------------------------------------------------------

def _grow(flux, overlap, graph):
    """Steps whose page calls come right before them: room reserved, a row forked, what a sparse request does not need released, the pool
    compacted, each directly followed by a decode.  Returns outputs, tables and pools."""
    Hq, Hkv, page, S, W, modes = 8, 2, 16, 16, 32, (1, 0, 1)
    plan = _plan(flux, Hq, Hkv, S, W, modes, 400)
    n_pages = 70
    pools = [_rows(31 + z, n_pages * page, Hkv).view(n_pages, page, Hkv, 128) for z in range(2)]
    table, refs = torch.full((3, 24), -1, dtype=torch.int32, device=DEV), torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    pages, pool = flux.Pages(*pools, table), flux.PagePool(table, refs, pools)
    lens = _dev([90, 200, 15])
    plan.flux_pages_reserve(pool, None, _dev([0, 0, 0]), lens)
    rope = flux.Rope(_inv_freq(128), device=DEV)
    x = _rows(5, 3, Hq + 2 * Hkv)
    out, nxt, edge, zero = torch.zeros(3, Hq, 128, dtype=torch.bfloat16, device=DEV), lens.clone(), _dev([0]), _dev([0])
    one, sink, top, two = _dev([1]), _dev([S]), _dev([2 ** 31 - 1]), _dev([2])
    found = []
    plan.flux_plan_set_launch_overlap(overlap)

    def step():
        torch.add(lens, 1, out=nxt)
        torch.sub(nxt[1:2], W, out=edge)
        lens.copy_(nxt)
        plan.flux_pages_release(pool, one, sink, edge)
        plan.flux_pages_reserve(pool, None, nxt - 1, nxt)
        plan.flux_attn_decode_step_paged(0, 3, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], pages, nxt, rope=rope, out=out)

    run = step
    if graph:
        keep = [t.clone() for t in (*pools, table, refs, lens)]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for t, s in zip((*pools, table, refs, lens), keep):
            t.copy_(s)
        run = g.replay
    for i in range(40):
        run()
        found.append(out.clone())
        if i % 10 == 5:
            q = _rows(i, 3, Hq)
            plan.flux_pages_fork(pool, zero, two, lens[:1])
            torch.cuda.synchronize()
            lens[2] = lens[0]
            plan.flux_pages_compact(pool)
            found.append(plan.flux_attn_decode_paged(0, 3, q, pages, lens))
            plan.flux_pages_release(pool, two, _dev([100]), top)                # (below its length: those positions count as masked)
            found.append(plan.flux_attn_decode_paged(0, 3, q, pages, lens))
            assert plan.flux_plan_status(raise_on_flag=False) in (0, flux.FLUX_STATUS_BAD_PAGE)
            plan.flux_pages_fork(pool, zero, two, lens[:1])
            found.append(plan.flux_attn_decode_paged(0, 3, q, pages, lens))
    assert plan.flux_plan_status() == 0
    return [torch.stack(found), table.clone(), refs.clone(), *(_bits(p.nan_to_num()) for p in pools)]


def test_decodes_right_behind_page_calls_with_overlap(flux):
    want = _grow(flux, False, False)
    for overlap, graph in ((True, False), (False, True), (True, True)):
        assert all(torch.equal(a, b) for a, b in zip(_grow(flux, overlap, graph), want)), (overlap, graph)


# ---- entries that a fork must not take or count --------------------------------------------------------------------------

def _book(flux, table, n_pages, page=16, refs=None):
    """A pool of one slab over this table, on the device and in the oracle."""
    table = np.asarray(table, dtype=np.int32)
    refs = np.bincount(table[(table >= 0) & (table < n_pages)], minlength=n_pages) if refs is None else refs
    data = _rows(n_pages, n_pages * page, 1).view(n_pages, page, 1, 128)
    t, r = _dev(table), _dev(refs)
    return flux.PagePool(t, r, [data]), paged.Pool(table, refs, _bits(data).cpu().numpy()[None], page)


def _same(flux, plan, pool, o):
    bits = plan.flux_plan_status(raise_on_flag=False)
    want = (flux.FLUX_STATUS_BAD_PAGE if o.bad_page else 0) | (flux.FLUX_STATUS_BAD_LENGTH if o.bad_length else 0) | (flux.FLUX_STATUS_NO_PAGES if o.no_pages else 0)
    o.bad_page = o.bad_length = o.no_pages = False
    assert bits == want and np.array_equal(pool.table.cpu().numpy(), o.table) and np.array_equal(pool.refs.cpu().numpy(), o.refs)
    assert np.array_equal(_bits(pool.slabs[0]).cpu().numpy(), o.data[0])
    return bits


@pytest.mark.parametrize("entry", [30, -2, -2 ** 31, 2 ** 31 - 1, 29])            # outside the pool; 29 is in it and free
def test_fork_of_entries_that_are_not_counted(flux, entry):
    """In a source row, in a row that is replaced, in both; taken by several rows at once; a fork that follows is served as if they had never
    been there, and so is a reservation, which may hand page 29 out."""
    plan, P = _plan(flux, 1, 1), 30

    def fresh(*places):
        table = np.full((7, 40), -1)
        table[0, :3], table[1, :2], table[2, :4], table[3, 35:37] = [0, 1, 2], [3, 4], [0, 1, 5, 6], [7, 8]
        refs = np.bincount(table[table >= 0], minlength=P)
        for place in places:
            table[place] = entry
        return _book(flux, table, P, refs=refs)

    def fork(b, src, dst, n):
        plan.flux_pages_fork(b[0], _dev(src), _dev(dst), _dev(n))
        b[1].fork(src, dst, n)
        return _same(flux, plan, *b)

    bad = flux.FLUX_STATUS_BAD_PAGE
    b = fresh((0, 1))
    assert fork(b, [0], [4], [48]) == bad                      # from a source
    assert fork(b, [4], [5], [48]) == 0
    b = fresh((0, 1))
    assert fork(b, [0, 0, 0, 0], [3, 4, 5, 6], [48, 48, 20, 16]) == bad          # by several at once (the last takes one page only)
    b = fresh((1, 1), (1, 39))
    assert fork(b, [0], [1], [48]) == bad                      # replaced
    assert fork(b, [2], [1], [64]) == 0
    b = fresh((0, 2), (1, 2), (3, 36), (3, 2))
    assert fork(b, [1, 0, 3], [0, 1, 3], [640, 640, 640]) == bad                 # rows change places, one takes itself
    if entry == 29:                                            # the free page is not held by anyone now: it is handed out once
        rows, a, e = [4, 5], [0, 0], [16 * 10, 16 * 11]
        got = plan.flux_pages_reserve(b[0], _dev(rows), _dev(a), _dev(e))
        assert got.tolist() == b[1].reserve(rows, a, e) == [1, 1]
        assert _same(flux, plan, *b) == 0
        held = b[1].table[b[1].table >= 0]
        assert len(set(held[held >= 9])) == (held >= 9).sum() and 29 in held
    assert fork(b, [0, 1], [1, 0], [640, 640]) == 0


def test_fork_of_pages_in_several_columns(flux):
    """A page held in columns that different CTAs own, its count going down and up in one call: it stays counted throughout."""
    plan = _plan(flux, 1, 1)
    table = np.full((40, 200), -1)
    for r in range(39):
        table[r, [(r * 5) % 200, (r * 5 + 67) % 200, (r * 5 + 133) % 200]] = r % 13
    b = _book(flux, table, 20)
    for turn in range(5):
        order = np.random.default_rng(turn).permutation(40).tolist()
        plan.flux_pages_fork(b[0], _dev(order), _dev(list(range(40))), _dev([200 * 16] * 40))
        b[1].fork(order, list(range(40)), [200 * 16] * 40)
        assert _same(flux, plan, *b) == 0


# ---- counters after a timeout --------------------------------------------------------------------------------------------

def test_a_timeout_clears_the_paged_decodes_counters_too(flux):
    """flux_plan_status brings all arrival counters back to zero once a wait has expired, those of the groups of CTAs among them (the last part
    of the workspace: 512 + max_batch words here)."""
    B, n, page = 64, 30000, 64
    plan = _plan(flux, 16, 1, modes=(1,) * B, max_ctx=n)
    pools = [_rows(41 + z, n, 1) for z in range(2)]
    pools = [torch.cat([x, x[:-(-n // page) * page - n]]).view(-1, page, 1, 128) for x in pools]
    pages = flux.Pages(*pools, _dev(np.arange(len(pools[0]))[None]))
    q = _rows(43, 1, 16)
    want = plan.flux_attn_decode_paged(0, 1, q, pages, _dev([n]))
    counters = plan.workspace[-4 * (512 + B):]
    assert not counters.any()
    counters.view(torch.int32).fill_(3)                        # (as a kernel that had left early would)
    plan.flux_debug_wait_probe(2_000_000)
    with pytest.raises(flux.FluxError) as e:
        plan.flux_plan_status()
    assert e.value.code == flux.FLUX_E_DEVICE_TIMEOUT and not counters.any()
    assert torch.equal(plan.flux_attn_decode_paged(0, 1, q, pages, _dev([n])), want) and plan.flux_plan_status() == 0


# ---- tables of more rows than a call lists -------------------------------------------------------------------------------

def test_rows_beyond_those_a_call_lists(flux):
    """9000 rows of 70 columns: the scratch has room for 4096 listed rows, wherever in the table they are.  What lies behind it stays as it was."""
    plan, rows, cols = _plan(flux, 1, 1), 9000, 70
    b = _book(flux, np.full((rows, cols), -1), 30000)
    pool, o = b
    guarded = torch.full((pool._scratch.numel() + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    pool.struct.scratch = guarded.data_ptr()
    some = np.random.default_rng(1).permutation(rows)[:4096]
    some[:2] = [rows - 1, 4096] if not {rows - 1, 4096} & set(some[2:].tolist()) else some[:2]
    a, e = [0] * 4096, [1 + 16 * int(i % 7) for i in range(4096)]
    e[-1] = 70 * 16
    got = plan.flux_pages_reserve(pool, _dev(some), _dev(a), _dev(e))
    assert got.tolist() == o.reserve(some.tolist(), a, e)
    _same(flux, plan, *b)
    plan.flux_pages_fork(pool, _dev(some[:1000]), _dev(some[3000:4000]), _dev(e[:1000]))
    o.fork(some[:1000].tolist(), some[3000:4000].tolist(), e[:1000])
    _same(flux, plan, *b)
    more = [x + 1 for x in e[:1000]]
    got = plan.flux_pages_reserve(pool, _dev(some[3000:4000]), _dev(e[:1000]), _dev(more))
    assert got.tolist() == o.reserve(some[3000:4000].tolist(), e[:1000], more)
    _same(flux, plan, *b)
    to, used = plan.flux_pages_compact(pool)
    want, n = o.compact()
    assert np.array_equal(to.cpu().numpy(), want) and int(used) == n
    _same(flux, plan, *b)
    assert (guarded[-4096:] == 0x5a).all()


# ---- infinities in K and non-finite query rows ---------------------------------------------------------------------------

def _near(q, k, v, out, what):
    """One head's row against the formula in 64 bits.  With weights p_j, A = sum p_j |v_j|: half a step of the output 2^-8 |ref|, weights as two
    bf16 numbers 2^-16 A, and weights off by a factor 1 + D, D = 2^-20 + 2^-16 of the largest score's sum of magnitudes (fp32 sums)."""
    s = k @ q / np.sqrt(128)
    p = np.exp(s - s.max())
    p /= p.sum()
    ref, A = p @ v, p @ np.abs(v)
    d = 2.0 ** -20 + 2.0 ** -16 * (np.abs(k) @ np.abs(q)).max() / np.sqrt(128)
    assert (np.abs(out - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * A + 2 * d * A).all(), what


@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("ctx", [200, 9000])
def test_a_non_finite_key_entry_by_the_sign_of_its_products(flux, ctx, value):
    Hq, Hkv, page, at, ch = 8, 2, 32, 121, 7
    plan = _plan(flux, Hq, Hkv, max_ctx=ctx)
    n_pages = -(-ctx // page)
    order = np.random.default_rng(ctx).permutation(n_pages)
    k, v = (_rows(51 + z, n_pages * page, Hkv) for z in range(2))
    q = _rows(53, 1, Hq)
    q[0, :, ch] = torch.tensor([1.0, -1.0] * 4, device=DEV)
    k[at, 1, ch] = value
    pools = [torch.empty_like(x).view(n_pages, page, Hkv, 128) for x in (k, v)]
    for pool, x in zip(pools, (k, v)):
        pool[torch.from_numpy(order).to(DEV)] = x.view(n_pages, page, Hkv, 128)
    out = plan.flux_attn_decode_paged(0, 1, q, flux.Pages(*pools, _dev(order[None])), _dev([ctx]))[0].double().cpu().numpy()
    q64, k64, v64 = q[0].double().cpu().numpy(), k.double().cpu().numpy()[:ctx], v.double().cpu().numpy()[:ctx]
    others = np.arange(ctx) != at
    for h in range(Hq):
        g = h // 4
        if g == 0:
            _near(q64[h], k64[:, 0], v64[:, 0], out[h], "head %d" % h)
        elif value != value or q64[h, ch] * value > 0:
            assert not np.isfinite(out[h]).any(), h
        else:                                                  # weight 0: as if the position were masked
            _near(q64[h], k64[others, 1], v64[others, 1], out[h], "head %d" % h)
    assert plan.flux_plan_status() == 0


def test_a_row_whose_scores_are_all_minus_infinity_is_zero(flux):
    plan = _plan(flux, 4, 1, max_ctx=100)
    k, v, q = _rows(61, 112, 1), _rows(62, 112, 1), _rows(63, 1, 4)
    k[:, 0, 3] = -INF
    q[0, :, 3] = torch.tensor([1.0, -1.0, 2.0, 0.5], device=DEV)
    out = plan.flux_attn_decode_paged(0, 1, q, flux.Pages(k.view(7, 16, 1, 128), v.view(7, 16, 1, 128), _dev(np.arange(7)[None])), _dev([100]))[0]
    assert (out[[0, 2, 3]] == 0).all() and not torch.isfinite(out[1]).any() and plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (16, 1)])
@pytest.mark.parametrize("step", [False, True])
def test_a_non_finite_query_entry_concerns_its_row_alone(flux, Hq, Hkv, step):
    ctx, page = 3000, 64
    plan = _plan(flux, Hq, Hkv, max_ctx=ctx)
    n_pages = -(-ctx // page)
    k, v, q = _rows(71, n_pages * page, Hkv), _rows(72, n_pages * page, Hkv), _rows(73, 1, Hq)
    rope = flux.Rope(np.zeros(64), device=DEV) if step else None                # angles of 0: rows as they are
    q[0, 1, 9], q[0, 4, 100], q[0, 6, 0] = NAN, INF, -INF
    pages = flux.Pages(k.view(n_pages, page, Hkv, 128), v.view(n_pages, page, Hkv, 128), _dev(np.arange(n_pages)[None]))
    if step:
        out = plan.flux_attn_decode_step_paged(0, 1, q, k[ctx - 1:ctx].clone(), v[ctx - 1:ctx].clone(), pages, _dev([ctx]), rope=rope)
    else:
        out = plan.flux_attn_decode_paged(0, 1, q, pages, _dev([ctx]))
    out, q64, k64, v64 = out[0].double().cpu().numpy(), q[0].double().cpu().numpy(), k[:ctx].double().cpu().numpy(), v[:ctx].double().cpu().numpy()
    for h in range(Hq):
        if h in (1, 4, 6):
            assert not np.isfinite(out[h]).any(), h
        else:
            _near(q64[h], k64[:, h // (Hq // Hkv)], v64[:, h // (Hq // Hkv)], out[h], "head %d" % h)
    assert plan.flux_plan_status() == 0


# ---- a row released twice in one call ------------------------------------------------------------------------------------

def test_release_applies_every_listing_of_a_row(flux):
    plan = _plan(flux, 1, 1)
    b = _book(flux, [[0, 1, 2, 3, 4, 5], [0, 1, 6, 7, -1, -1]], 10)
    rows, begin, end = [0, 1, 0, 0, 1], [0, 16, 40, 64, 16], [16, 48, 80, 2 ** 31 - 1, 33]      # pages 0; 1, 6; 3, 4; 4, 5; 1
    plan.flux_pages_release(b[0], _dev(rows), _dev(begin), _dev(end))
    b[1].release(rows, begin, end)
    assert b[1].table.tolist() == [[-1, 1, 2, -1, -1, -1], [0, -1, -1, 7, -1, -1]] and _same(flux, plan, *b) == 0
    assert b[1].refs.tolist() == [1, 1, 1, 0, 0, 0, 0, 1, 0, 0]
