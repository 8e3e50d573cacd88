"""GPU parity of the paged KV cache: norm and rotation, store and load, decode over pages, bookkeeping; against the fp64 oracle.

Norm and rotation: an entry y = inv (x_a c w_a - x_b s w_b) is off by at most
    2^-8 |y|            bf16 output (half a step)
  + 2^-17 (|y_a| + |y_b|)  with |y_a| + |y_b| what the pair would add up to without cancelling: sum of 128 squares and its root
                        2^-18 (128 additions of 2^-24, halved by the root), angle pi 2^-24 (fp32 fraction of half a turn), sine and cosine
                        2^-22, a handful of products at 2^-24 each; the fraction of a turn itself 2^-33.
What is stored and loaded is compared exactly.

Decode outputs: with p_j the softmax weights and A = sum_j p_j |v_j|, an element is off by at most
    2^-8 |ref|                       bf16 output
  + 2^-16 A                          weights as two bf16 numbers, each rounded by half a step
  + 2 D A                            weights off by a factor 1 + D: D = 2^-20 (log2, ex2, reciprocal, fp32 sums and rescaling by at most a few
                                     dozen factors of 2^-24 each) + 2^-16 of the largest sum_d |q_d k_d| scale (128 fp32 additions); where
                                     the call turns the query rows itself, the error of such a row comes to that: 2^-17 (|y_a| + |y_b|) as above
                                     and 2^-16 of y (two bf16 numbers)
"""
import numpy as np
import pytest
import torch

from oracle import kvq, paged

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAN = float("nan")


@pytest.fixture(scope="module")
def flux():
    from paper_2604_07394_b200 import build, flux as f
    build.build()
    f.load()
    return f


def _dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _cum(x):
    return [0] + np.cumsum(x).tolist()


def _plan(flux, Hq, Hkv, S=4, W=8, modes=(1,), max_ctx=1 << 20, **kw):
    plan = flux.Plan(flux.make_config(1, Hq, Hkv, S, W, len(modes), max_ctx, **kw), DEV)
    plan.flux_router_apply(mask=np.array([[m] for m in modes], dtype=np.uint8))
    return plan


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(gen, n, heads):
    x = torch.randn(n, heads, 128, generator=gen, device=DEV)
    big = torch.ones(128, device=DEV)
    big[5::31] = 6.0                       # a few large channels, as keys have
    return (x * big).to(torch.bfloat16)


def _f64(x):
    return x.double().cpu().numpy()


def _inv_freq(rot, theta=1e4):
    return theta ** (-np.arange(0, rot, 2) / max(rot, 1))


def _check_turned(got, ref, mag, what=""):
    got = _f64(got)
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -17 * mag
    assert np.isfinite(got).all() and (np.abs(got - ref) <= tol).all(), "%s: %.2f of the tolerance" % (what, (np.abs(got - ref) / np.maximum(tol, 1e-300)).max())


def _check_decode(q, k, v, out, what="", turned=None):
    """q, out [Hq][128], k, v [m][Hkv][128], fp64; turned: |y_a| + |y_b| of query rows that the call has normed and rotated."""
    ref, A, mag, _ = kvq.attend(q, k, v, 1 / np.sqrt(128))
    d = 2.0 ** -20 + 2.0 ** -16 * mag
    if turned is not None:
        d = d + kvq.attend(2.0 ** -17 * turned + 2.0 ** -16 * np.abs(q), k, v, 1 / np.sqrt(128))[2]
    tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * A + 2 * d[:, None] * A
    err = np.abs(out - ref)
    assert np.isfinite(out).all() and (err <= tol).all(), "%s: %.2f of the tolerance" % (what, (err / np.maximum(tol, 1e-300)).max())


# ---- norm and rotation ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("Hq,Hkv,rot,pairs,norm,offset,scale", [
    (32, 8, 128, False, True, 0.0, 1.0), (28, 4, 64, True, True, 1.0, 1.0), (7, 7, 96, False, False, 0.0, 1.25), (1, 1, 16, False, True, 0.0, 1.0),
    (16, 1, 128, True, False, 0.0, 1.0), (36, 3, 0, False, True, 1.0, 1.0), (3, 3, 112, True, True, 0.0, -0.5), (5, 1, 48, False, False, 0.0, 1.0)])
def test_rows_against_the_oracle(flux, Hq, Hkv, rot, pairs, norm, offset, scale):
    gen = _gen(rot + Hq)
    plan = _plan(flux, Hq, Hkv)
    pos = [0, 1, 2, 77, 4095, 131071, 1000003, 2 ** 31 - 1, -5, 0, 12345678]
    n = len(pos)
    fused = _rows(gen, n + 2, Hq + 2 * Hkv)
    q, k = fused[:n, :Hq], fused[:n, Hq:Hq + Hkv]
    w = [(torch.randn(128, generator=gen, device=DEV) + 1 - offset).to(torch.bfloat16) if norm else None for _ in "qk"]
    f = _inv_freq(rot, 5e5)
    rope = flux.Rope(f, q_weight=w[0], k_weight=w[1], eps=1e-5, interleaved=pairs, scale=scale, weight_offset=offset, device=DEV)
    out = plan.flux_qk_norm_rope(rope, q, k, _dev(pos))
    for x, got, weight in zip((q, k), out, w):
        ref, mag = paged.turned(_f64(x), pos, f, None if weight is None else _f64(weight), 1e-5, offset, scale, pairs)
        _check_turned(got, ref, mag)
    # one alone; in place, strided, the neighbours untouched
    only = plan.flux_qk_norm_rope(rope, None, k, _dev(pos))
    assert only[0] is None and torch.equal(only[1], out[1])
    before = fused.clone()
    plan.flux_qk_norm_rope(rope, q, k, _dev(pos), q_out=q, k_out=k)
    assert torch.equal(fused[:n, :Hq], out[0]) and torch.equal(fused[:n, Hq:Hq + Hkv], out[1])
    assert torch.equal(fused[n:], before[n:]) and torch.equal(fused[:, Hq + Hkv:], before[:, Hq + Hkv:])
    assert plan.flux_qk_norm_rope(rope, q, k, _dev([]))[0].shape == (0, Hq, 128)
    assert plan.flux_plan_status() == 0


@pytest.mark.parametrize("n", [1, 3, 200, 5000])
def test_a_row_does_not_depend_on_how_many_there_are(flux, n):
    """Few rows are dealt to several warps, many to one each."""
    gen = _gen(n)
    plan = _plan(flux, 28, 4)
    q, k, pos = _rows(gen, n, 28), _rows(gen, n, 4), torch.randint(0, 200000, (n,), generator=gen, device=DEV, dtype=torch.int32)
    w = torch.rand(128, generator=gen, device=DEV).to(torch.bfloat16)
    rope = flux.Rope(_inv_freq(128), q_weight=w, k_weight=w, device=DEV)
    out = plan.flux_qk_norm_rope(rope, q, k, pos)
    for i in {0, n // 2, n - 1}:
        one = plan.flux_qk_norm_rope(rope, q[i:i + 1], k[i:i + 1], pos[i:i + 1])
        assert torch.equal(one[0][0], out[0][i]) and torch.equal(one[1][0], out[1][i])


def test_zero_rows_and_non_finite_entries_stay_in_their_head(flux):
    gen = _gen(3)
    plan = _plan(flux, 4, 2)
    q, k = _rows(gen, 3, 4), _rows(gen, 3, 2)
    q[0, 1] = 0
    q[1, 2, 5], q[2, 3, 100] = NAN, float("inf")
    w = torch.ones(128, dtype=torch.bfloat16, device=DEV)
    rope = flux.Rope(_inv_freq(128), q_weight=w, k_weight=w, device=DEV)
    out, _ = plan.flux_qk_norm_rope(rope, q, k, _dev([1, 2, 3]))
    fin = torch.isfinite(out).all(-1)
    assert (out[0, 1] == 0).all() and not fin[1, 2] and not fin[2, 3] and int(fin.sum()) == 10


# ---- store and load --------------------------------------------------------------------------------------------------

class Rig:
    """Pools whose every position that no request keeps is NaN, requests anywhere in them."""

    def __init__(self, flux, Hq, Hkv, S, W, modes, ctx, page, seed=1, spare=3, room=0, rows=None, **kw):
        self.flux, self.Hq, self.Hkv, self.S, self.W, self.modes, self.ctx, self.page = flux, Hq, Hkv, S, W, modes, ctx, page
        self.plan = _plan(flux, Hq, Hkv, S, W, modes, max(max(ctx) + room, 1), **kw)
        gen = self.gen = _gen(seed)
        rng = np.random.default_rng(seed)
        cols = max(-(-(max(ctx) + room) // page), 1)
        self.table_host = np.full((len(ctx), cols), -1, dtype=np.int32)
        self.keep = [kvq.kept(n, m == 1, S, W) for n, m in zip(ctx, modes)]
        for b, keep in enumerate(self.keep):
            self.table_host[b, np.unique(keep // page)] = 0
        count = int((self.table_host == 0).sum())
        self.n_pages = count + spare
        self.table_host[self.table_host == 0] = rng.permutation(self.n_pages)[:count]
        self.k, self.v = (torch.full((self.n_pages, page, Hkv, 128), NAN, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        self.rows = []                                        # kept K, V rows of every request
        for b, keep in enumerate(self.keep):
            kv = [_rows(gen, len(keep), Hkv), _rows(gen, len(keep), Hkv)] if rows is None else rows(b, len(keep), gen)
            self.rows.append(kv)
            at = self.slots(b, keep)
            for pool, x in zip((self.k, self.v), kv):
                pool.view(-1, Hkv, 128)[at] = x
        self.table = torch.from_numpy(self.table_host).to(DEV)
        self.pages = flux.Pages(self.k, self.v, self.table)

    def slots(self, b, pos):
        pos = np.asarray(pos)
        return torch.from_numpy(self.table_host[b, pos // self.page].astype(np.int64) * self.page + pos % self.page).to(DEV)

    def decode(self, q, **kw):
        return self.plan.flux_attn_decode_paged(0, len(self.ctx), q, self.pages, _dev(self.ctx), **kw)

    def check(self, q, out, what="", turned=None):
        q = _f64(q) if isinstance(q, torch.Tensor) else q
        for b, (k, v) in enumerate(self.rows):
            if len(k) == 0:
                assert (out[b] == 0).all(), what
            else:
                _check_decode(q[b], _f64(k), _f64(v), _f64(out[b]), "%s request %d of %d tokens" % (what, b, self.ctx[b]),
                              None if turned is None else turned[b])


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (5, 5), (16, 1)])
def test_store_then_load(flux, page, Hq, Hkv):
    gen = _gen(page + Hq)
    new, past = [0, 1, 40, 17, 0, 300, 2, page], [0, 0, 7, 15, 9, page - 1, 2 * page, page]
    ends = [n + p for n, p in zip(new, past)]
    r = Rig(flux, Hq, Hkv, 4, 8, [1] * len(new), ends, page, rows=lambda b, n, g: [torch.full((n, Hkv, 128), 7.0, device=DEV).bfloat16()] * 2)
    total = sum(new) + 3                                      # rows behind the last request
    fused = _rows(gen, total, Hq + 2 * Hkv)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    rope = flux.Rope(_inv_freq(64), k_weight=torch.rand(128, generator=gen, device=DEV).bfloat16(), device=DEV)
    at = np.concatenate([p + np.arange(n) for n, p in zip(new, past)] + [[0, 0, 0]])
    want_q, want_k = r.plan.flux_qk_norm_rope(rope, q, k, _dev(at))
    k0, v0 = r.k.clone(), r.v.clone()
    q_out, k_out = torch.full((total, Hq, 128), 3.0, device=DEV).bfloat16(), torch.full((total, Hkv, 128), 3.0, device=DEV).bfloat16()
    got = r.plan.flux_paged_store(r.pages, k, v, _dev(_cum(new)), _dev(past), rope=rope, q=q, q_out=q_out, k_out=k_out)
    n = sum(new)
    assert got is q_out and torch.equal(q_out[:n], want_q[:n]) and torch.equal(k_out[:n], want_k[:n])
    assert (q_out[n:] == 3).all() and (k_out[n:] == 3).all()
    for b, (a, e) in enumerate(zip(_cum(new), _cum(new)[1:])):
        s = r.slots(b, past[b] + np.arange(new[b]))
        k0.view(-1, Hkv, 128)[s], v0.view(-1, Hkv, 128)[s] = want_k[a:e], v[a:e]
    assert torch.equal(r.k.view(torch.int16), k0.view(torch.int16)) and torch.equal(r.v.view(torch.int16), v0.view(torch.int16))
    # without a rope the rows as they are; the whole of every request read back, and a part
    r.plan.flux_paged_store(r.pages, k, v, _dev(_cum(new)), _dev(past))
    lk, lv = r.plan.flux_paged_load(r.pages, _dev(ends), _dev(_cum(ends)), _dev([0] * len(new)), sum(ends))
    for b, (a, e) in enumerate(zip(_cum(new), _cum(new)[1:])):
        z = _cum(ends)[b]
        assert (lk[z:z + past[b]] == 7).all() and (lv[z:z + past[b]] == 7).all()
        assert torch.equal(lk[z + past[b]:z + ends[b]], k[a:e]) and torch.equal(lv[z + past[b]:z + ends[b]], v[a:e])
    part = torch.full((9, Hkv, 128), 5.0, device=DEV).bfloat16()
    pv = part.clone()
    r.plan.flux_paged_load(r.pages, _dev(ends), _dev([2, 2, 2, 5, 5, 5, 5, 5, 5]), _dev([0, 0, 10, 0, 0, 0, 0, 0]), 9, part, pv)
    a = _cum(new)[2] + 3
    assert torch.equal(part[2:5], k[a:a + 3]) and torch.equal(pv[2:5], v[a:a + 3]) and (part[[0, 1, 5, 6, 7, 8]] == 5).all()
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv,page,rot,pairs", [(32, 8, 16, 128, False), (28, 4, 64, 64, True), (7, 7, 32, 96, False), (9, 3, 128, 0, False)])
def test_many_rows_are_stored_like_few(flux, Hq, Hkv, page, rot, pairs):
    """From some thousand rows on a warp takes whole rows; results are those of calls with a few rows each.  Sparse requests have dropped
    pages, there are rows before, between and behind the requests' own, and one request's entries cannot be."""
    modes, new, past = [1, 0, 1, 0, 1, 1], [1500, 2900, 0, 1111, 1, 900], [0, 100, 5, 0, 3000, 17]
    ends = [n + p for n, p in zip(new, past)]
    rigs = [Rig(flux, Hq, Hkv, 40, 300, modes, ends, page, seed=3) for _ in range(2)]
    gen = _gen(rot)
    starts = [3 + x for x in _cum(new)]
    total = starts[-1] + 60
    fused = _rows(gen, total, Hq + 2 * Hkv)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    w = [torch.rand(128, generator=gen, device=DEV).bfloat16() for _ in "qk"]
    rope = flux.Rope(_inv_freq(rot), q_weight=w[0], k_weight=w[1], interleaved=pairs, device=DEV)
    for r in rigs:
        r.table[5, 3:5] = r.n_pages + 7
    outs = [[torch.full((total, h, 128), 2.0, device=DEV).bfloat16() for h in (Hq, Hkv)] for _ in rigs]
    a, b = rigs
    a.plan.flux_paged_store(a.pages, k, v, _dev(starts), _dev(past), rope=rope, q=q, q_out=outs[0][0], k_out=outs[0][1])
    for i in range(0, total, 200):                            # the same in pieces of 200 rows
        e = min(i + 200, total)
        cut = [min(max(x, i), e) - i for x in starts]
        at = [p + max(i - x, 0) for p, x in zip(past, starts)]
        b.plan.flux_paged_store(b.pages, k[i:e], v[i:e], _dev(cut), _dev(at), rope=rope, q=q[i:e], q_out=outs[1][0][i:e], k_out=outs[1][1][i:e])
    for x, y in zip([a.k, a.v] + outs[0], [b.k, b.v] + outs[1]):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    for x in outs[0]:
        assert (x[:3] == 2).all() and (x[starts[-1]:] == 2).all() and int((x == 2).all(-1).sum()) == 63 * x.shape[1]
    for r in rigs:
        assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE
    # and they are what the definition says, on a sample of rows
    for i in (3, 777, 1502, 4500, 6000, starts[-1] - 1):
        req = max(j for j in range(6) if starts[j] <= i and new[j])
        at = past[req] + i - starts[req]
        ref, mag = paged.turned(_f64(q[i:i + 1]), [at], _inv_freq(rot), _f64(w[0]), pairs=pairs)
        _check_turned(outs[0][0][i:i + 1], ref, mag, "row %d" % i)


def test_dropped_pages_take_no_rows_and_give_zeros(flux):
    r = Rig(flux, 4, 2, 20, 40, [0], [500], 16)
    x = _rows(r.gen, 500, 2)
    r.plan.flux_paged_store(r.pages, x, x, _dev([0, 500]), _dev([0]))
    k, v = r.plan.flux_paged_load(r.pages, _dev([500]), _dev([0, 500]), _dev([0]), 500)
    held = torch.from_numpy(r.table_host[0][np.arange(500) // 16] >= 0).to(DEV)
    assert torch.equal(k[held], x[held]) and torch.equal(v[held], x[held]) and (k[~held] == 0).all() and int((~held).sum()) > 400
    assert r.plan.flux_plan_status() == 0


def test_store_and_load_refusals(flux):
    r = Rig(flux, 4, 2, 4, 8, [1, 1], [30, 20], 16)
    x = _rows(r.gen, 90, 2)
    before = [r.k.clone(), r.v.clone()]

    def flagged(call, bits):
        call()
        assert r.plan.flux_plan_status(raise_on_flag=False) == bits
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, (r.k, r.v)))

    st = lambda rows, pos, pages=r.pages: (lambda: r.plan.flux_paged_store(pages, x, x, _dev(rows), _dev(pos)))  # noqa: E731
    bad = flux.FLUX_STATUS_BAD_LENGTH
    flagged(st([0, 40, 40], [0, 0]), bad)                     # past max_context
    flagged(st([0, 0, 91], [0, 0]), bad)                      # past the rows given
    flagged(st([10, 5, 5], [0, 0]), bad)
    flagged(st([0, 1, 1], [-1, 0]), bad)
    flagged(st([-3, 0, 0], [0, 0]), bad)
    flagged(st([0, 1, 1], [2 ** 31 - 1, 0]), bad)
    for entry in (r.n_pages, -2, 2 ** 31 - 1):
        wrong = flux.Pages(r.k, r.v, torch.full_like(r.table, entry))
        flagged(st([0, 5, 6], [0, 0], wrong), flux.FLUX_STATUS_BAD_PAGE)
        flagged(lambda: r.plan.flux_paged_load(wrong, _dev([30, 20]), _dev([0, 5, 6]), _dev([0, 0]), 6), flux.FLUX_STATUS_BAD_PAGE)
    for ctx, rows, pos in (([30, 20], [0, 31, 31], [0, 0]), ([30, 20], [0, 3, 3], [28, 0]), ([-1, 20], [0, 1, 1], [0, 0]), ([31, 20], [0, 1, 1], [0, 0])):
        flagged(lambda: r.plan.flux_paged_load(r.pages, _dev(ctx), _dev(rows), _dev(pos), 31), bad)
    rope = flux.Rope(_inv_freq(128), device=DEV)
    odd = torch.zeros(90 * 256 + 8, dtype=torch.bfloat16, device=DEV)[1:1 + 90 * 256].view(90, 2, 128)
    q = _rows(r.gen, 90, 4)
    none, two = _dev([0, 1, 2]), _dev([0, 0])

    def wrong_rope(**kw):
        s = flux.Rope(_inv_freq(128), device=DEV)
        for name, value in kw.items():
            setattr(s.struct, name, value)
        return s

    for call, code in ((lambda: r.plan.flux_paged_store(r.pages, odd, x, none, two), flux.FLUX_E_INVALID_ARG),
                       (lambda: r.plan.flux_paged_store(r.pages, x, x, none, two, q=q), flux.FLUX_E_INVALID_ARG),
                       (lambda: r.plan.flux_paged_store(r.pages, x, x, none, two, rope=wrong_rope(rotary_dim=40)), flux.FLUX_E_UNSUPPORTED_SHAPE),
                       (lambda: r.plan.flux_paged_store(r.pages, x, x, none, two, rope=wrong_rope(rotary_dim=144)), flux.FLUX_E_UNSUPPORTED_SHAPE),
                       (lambda: r.plan.flux_paged_store(r.pages, x, x, none, two, rope=wrong_rope(eps=-1.0)), flux.FLUX_E_INVALID_ARG),
                       (lambda: r.plan.flux_paged_store(r.pages, x, x, none, two, rope=wrong_rope(freqs=None)), flux.FLUX_E_INVALID_ARG),
                       (lambda: r.plan.flux_paged_store(r.pages, x, x, none, two, rope=wrong_rope(scale=NAN)), flux.FLUX_E_INVALID_ARG),
                       (lambda: r.plan.flux_attn_decode_paged(1, 2, q, r.pages, two), flux.FLUX_E_INVALID_ARG)):
        with pytest.raises(flux.FluxError) as e:
            call()
        assert e.value.code == code
    three = flux.Pages(_rows(r.gen, 16, 3).view(1, 16, 3, 128), _rows(r.gen, 16, 3).view(1, 16, 3, 128), r.table)
    for call in (lambda: r.plan.flux_paged_store(r.pages, x, x[:5], none, two), lambda: r.plan.flux_paged_store(r.pages, x.float(), x, none, two),
                 lambda: r.plan.flux_paged_store(r.pages, x, x, none[:2], two), lambda: r.plan.flux_paged_store(r.pages, x, x, none, _dev([0, 0, 0])),
                 lambda: r.plan.flux_paged_store(three, x, x, none, two), lambda: r.plan.flux_paged_store(r.pages, x, x, none, two.long()),
                 lambda: r.plan.flux_qk_norm_rope(rope, q[:3], None, _dev([0] * 4)), lambda: r.plan.flux_qk_norm_rope(rope, q.cpu(), None, none),
                 lambda: r.plan.flux_qk_norm_rope(rope, x, None, none), lambda: r.decode(q[:1]), lambda: r.decode(q[:, :2]),
                 lambda: flux.Pages(r.k, r.v, r.table.cpu()), lambda: flux.Pages(r.k.cpu(), r.v, r.table)):
        with pytest.raises(ValueError):
            call()
    flagged(lambda: None, 0)


# ---- decode ----------------------------------------------------------------------------------------------------------

LENS = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 0, 255, 257, 300, 777]


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv,S,W", [(8, 2, 5, 33), (5, 5, 0, 1), (16, 1, 64, 64), (36, 3, 20, 100), (28, 4, 16, 32)])
def test_decode_over_every_length(flux, page, Hq, Hkv, S, W):
    modes = [i % 2 for i in range(len(LENS))] + [1 - i % 2 for i in range(len(LENS))]
    r = Rig(flux, Hq, Hkv, S, W, modes, LENS * 2, page, seed=page + Hq)
    q = _rows(r.gen, len(modes), Hq)
    out = r.decode(q)
    r.check(q, out)
    rec = r.plan.flux_debug_dispatch()
    assert [int(x[3]) for x in rec] == LENS * 2 and [int(x[0]) for x in rec] == modes
    wide = torch.full((len(modes), Hq + 3, 128), NAN, dtype=torch.bfloat16, device=DEV)
    wide[:, 1:1 + Hq] = q
    assert torch.equal(r.decode(wide[:, 1:1 + Hq]), out)      # query rows inside a wider projection output
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv,ctx", [(32, 8, [20000]), (28, 4, [9001, 4, 30000]), (16, 1, [40000, 1]), (8, 8, [5000, 17, 0, 8000]), (36, 3, [12345])])
def test_decode_split_over_many_ctas(flux, Hq, Hkv, ctx):
    for modes in ([1] * len(ctx), [i % 2 for i in range(len(ctx))]):
        r = Rig(flux, Hq, Hkv, 128, 2048, modes, ctx, 64, seed=sum(ctx))
        q = _rows(r.gen, len(ctx), Hq)
        out = r.decode(q)
        r.check(q, out)
        assert all(torch.equal(r.decode(q), out) for _ in range(3)) and r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv,ctx,page", [(4, 1, [30011], 16), (8, 1, [50000], 256), (11, 1, [7, 30000, 64], 64), (16, 1, [2600], 16), (16, 2, [33000], 32), (32, 2, [20000, 3, 20001], 128),
                                             (48, 3, [9999] * 2, 64)])
def test_decode_of_partials_added_up_in_groups(flux, Hq, Hkv, ctx, page):
    """Few KV heads of many query heads, so many CTAs share a segment; also with groups of CTAs that find no page."""
    r = Rig(flux, Hq, Hkv, 128, 2048, [1] * len(ctx), ctx, page, seed=sum(ctx))
    q = _rows(r.gen, len(ctx), Hq)
    out = r.decode(q)
    r.check(q, out)
    graph, lens = torch.cuda.CUDAGraph(), _dev(ctx)
    with torch.cuda.graph(graph):
        again = [r.plan.flux_attn_decode_paged(0, len(ctx), q, r.pages, lens) for _ in range(3)]
    graph.replay()
    graph.replay()
    assert all(torch.equal(x, out) for x in again) and r.plan.flux_plan_status() == 0
    long = int(np.argmax(ctx))
    cols = -(-ctx[long] // page)
    r.table[long, cols // 3:cols * 2 // 3] = -1
    out = r.decode(q)
    assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE
    stay = torch.ones(ctx[long], dtype=torch.bool, device=DEV)
    stay[cols // 3 * page:cols * 2 // 3 * page] = False
    _check_decode(_f64(q[long]), _f64(r.rows[long][0][stay]), _f64(r.rows[long][1][stay]), _f64(out[long]), "without a third")
    r.table[long] = -1
    out = r.decode(q)
    assert (out[long] == 0).all() and r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE


@pytest.mark.parametrize("B,Hq,Hkv", [(200, 8, 2), (1024, 4, 4), (300, 32, 4), (400, 32, 2)])
def test_decode_of_large_batches(flux, B, Hq, Hkv):
    rng = np.random.default_rng(B)
    r = Rig(flux, Hq, Hkv, 16, 40, [int(x) for x in rng.integers(0, 2, B)], [int(x) for x in rng.integers(0, 120, B)], 16, seed=B)
    q = _rows(r.gen, B, Hq)
    r.check(q, r.decode(q))
    assert r.plan.flux_plan_status() == 0


def test_decode_of_extreme_scores(flux):
    """A key that outweighs the others, scores far below -1e30, equal keys, and rows whose maximum rises tile after tile."""
    def rows(b, n, g):
        k, v = _rows(g, n, 2), _rows(g, n, 2)
        if b == 0:
            k[n // 2] *= 40
        elif b == 1:
            k[:] = torch.full_like(k, -1.0e17)
        elif b == 2:
            k[:] = k[0]
        else:
            k[:] = torch.linspace(0, 3, n, device=DEV)[:, None, None].bfloat16()
        return [k, v]

    r = Rig(flux, 8, 2, 4, 8, [1] * 4, [700, 50, 333, 900], 32, rows=rows)
    q = _rows(r.gen, 4, 8).abs()
    q[1] *= 1.0e13
    out = r.decode(q)
    keys = [_f64(k) for k, _ in r.rows]
    assert (np.einsum("hd,mhd->hm", _f64(q[1, ::4]), keys[1]).max() / np.sqrt(128)) < -1e30
    for b in (0, 2, 3):
        _check_decode(_f64(q[b]), keys[b], _f64(r.rows[b][1]), _f64(out[b]), str(b))
    # request 1: all scores of a head are equal (equal keys), so its output is the mean of V
    mean = np.repeat(_f64(r.rows[1][1]).mean(0), 4, axis=0)
    A = np.repeat(np.abs(_f64(r.rows[1][1])).mean(0), 4, axis=0)
    assert (np.abs(_f64(out[1]) - mean) <= 2.0 ** -8 * np.abs(mean) + 2.0 ** -18 * A).all()
    assert r.plan.flux_plan_status() == 0


def test_a_non_finite_kept_entry_stays_in_its_channel_or_head(flux):
    r = Rig(flux, 8, 2, 4, 8, [1, 1, 1], [300, 300, 300], 16)
    q = _rows(r.gen, 3, 8)
    want = r.decode(q)
    for pool, value, bad in ((r.v, float("inf"), lambda: out[0, 4:, 7]), (r.v, NAN, lambda: out[0, 4:, 7]), (r.k, NAN, lambda: out[0, 4:])):
        at = r.slots(0, [211])
        old = pool.view(-1, 2, 128)[at, 1, 7].clone()
        pool.view(-1, 2, 128)[at, 1, 7] = value
        out = r.decode(q)
        assert not bad().isfinite().any()
        bad()[:] = 0
        ref = want.clone()
        out, ref = ref, out                                   # the same entries of the other one
        bad()[:] = 0
        assert torch.equal(out, ref)
        pool.view(-1, 2, 128)[at, 1, 7] = old
    assert torch.equal(r.decode(q), want) and r.plan.flux_plan_status() == 0


def test_missing_pages_and_lengths_that_cannot_be(flux):
    r = Rig(flux, 8, 2, 16, 48, [1, 0, 1], [200, 200, 90], 16)
    q = _rows(r.gen, 3, 8)
    good = r.decode(q)
    table = r.table.clone()
    for entry in (-1, r.n_pages, -7, 2 ** 31 - 1):
        table[0, 3], table[1, 11], table[2, :] = entry, entry, entry
        out = r.plan.flux_attn_decode_paged(0, 3, q, flux.Pages(r.k, r.v, table), _dev(r.ctx))
        assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE
        # positions 48 .. 63, and 176 .. 191, count as masked; a request without any page: zeros
        for b, lost in ((0, 3), (1, 11)):
            stay = torch.from_numpy(r.keep[b] // 16 != lost).to(DEV)
            _check_decode(_f64(q[b]), _f64(r.rows[b][0][stay]), _f64(r.rows[b][1][stay]), _f64(out[b]), "request %d" % b)
        assert (out[2] == 0).all()
    for n in (201, 2 ** 31 - 1):
        out = r.plan.flux_attn_decode_paged(0, 3, q, r.pages, _dev([200, n, -3]))
        assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_LENGTH
        assert torch.equal(out[0], good[0]) and (out[1:] == 0).all()


def test_decode_touches_what_it_keeps(flux):
    r = Rig(flux, 8, 2, 20, 50, [1, 0, 0], [100, 300, 60], 32)
    bits = torch.zeros(3, 12, dtype=torch.int32, device=DEV)
    r.plan.flux_debug_touched(bits)
    r.decode(_rows(r.gen, 3, 8))
    r.plan.flux_debug_touched(None)
    words = bits.cpu().numpy().astype(np.uint32)
    for b in range(3):
        assert [p for p in range(384) if words[b, p // 32] >> (p % 32) & 1] == r.keep[b].tolist()


def test_pages_beyond_32_bits(flux):
    """5 GB pools: page offsets beyond 2^32 bytes, elements beyond 2^31."""
    page, Hkv, n_pages = 128, 8, 20000
    k, v = (torch.empty(n_pages, page, Hkv, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    assert k.numel() * 2 > 2 ** 32
    table = _dev([[n_pages - 1, 3, n_pages - 7], [16500, n_pages - 2, 17000]])
    pages = flux.Pages(k, v, table)
    plan = _plan(flux, 32, Hkv, modes=[1, 1], max_ctx=384)
    gen = _gen(5)
    x, y, ctx = _rows(gen, 600, Hkv), _rows(gen, 600, Hkv), [300, 300]
    plan.flux_paged_store(pages, x, y, _dev([0, 300, 600]), _dev([0, 0]))
    assert torch.equal(k[n_pages - 1], x[:128]) and torch.equal(v[17000, :44], y[556:])
    q = _rows(gen, 2, 32)
    out = plan.flux_attn_decode_paged(0, 2, q, pages, _dev(ctx))
    for b in range(2):
        _check_decode(_f64(q[b]), _f64(x[300 * b:300 * b + 300]), _f64(y[300 * b:300 * b + 300]), _f64(out[b]))
    lk, _ = plan.flux_paged_load(pages, _dev(ctx), _dev([0, 300, 600]), _dev([0, 0]), 600)
    assert torch.equal(lk, x)
    # a fork of request 0 writes on: its begun page, the last of the pool, is copied to page 0 and moves nowhere when compacted
    tab = torch.full((2, 4), -1, dtype=torch.int32, device=DEV)
    tab[0, :3] = table[0]
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[table[0].long()] = 1
    pool = flux.PagePool(tab, refs, [k, v])
    plan.flux_pages_fork(pool, _dev([0]), _dev([1]), _dev([300]))
    plan.flux_pages_reserve(pool, _dev([1]), _dev([300]), _dev([301]))
    assert tab[1].tolist() == [n_pages - 1, 3, 0, -1] and torch.equal(k[0, :44], x[256:300])
    to, used = plan.flux_pages_compact(pool)
    assert int(used) == 4 and tab.tolist() == [[2, 3, 1, -1], [2, 3, 0, -1]] and torch.equal(k[2], x[:128]) and torch.equal(v[1, :44], y[256:300])
    assert plan.flux_plan_status() == 0


# ---- the step in one launch ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("overlap", [False, True])
@pytest.mark.parametrize("Hq,Hkv,page,rot,pairs,norm", [(8, 2, 16, 128, False, True), (28, 4, 64, 64, True, True), (16, 1, 32, 96, False, False), (36, 3, 128, 0, False, True),
                                                        (5, 5, 16, None, False, False)])
def test_step_is_store_and_decode(flux, Hq, Hkv, page, rot, pairs, norm, overlap):
    lens = [n for n in LENS if n] + [0, 2000, 5000]
    modes = [(i * 7) % 3 % 2 for i in range(len(lens))]
    gen = _gen(page)
    w = [torch.rand(128, generator=gen, device=DEV).bfloat16() if norm else None for _ in "qk"]
    rope = None if rot is None else flux.Rope(_inv_freq(rot), q_weight=w[0], k_weight=w[1], interleaved=pairs, device=DEV)
    rigs = [Rig(flux, Hq, Hkv, 20, 100, modes, lens, page, seed=page) for _ in range(2)]
    fused = _rows(gen, len(lens), Hq + 2 * Hkv)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    a, b = rigs
    for r in rigs:                                            # the newest position is not there yet
        for i, n in enumerate(lens):
            if n:
                for pool in (r.k, r.v):
                    pool.view(-1, Hkv, 128)[r.slots(i, [n - 1])] = NAN
        r.plan.flux_plan_set_launch_overlap(overlap)
    live = [i for i, n in enumerate(lens) if n]
    start = _dev(_cum([1 if n else 0 for n in lens]))
    turned = a.plan.flux_paged_store(a.pages, k[live], v[live], start, _dev([max(n - 1, 0) for n in lens]), rope=rope, q=q[live] if rope else None)
    qr = torch.zeros(len(lens), Hq, 128, dtype=torch.bfloat16, device=DEV)
    qr[live] = turned if rope else q[live]
    want = a.decode(qr)
    got = b.plan.flux_attn_decode_step_paged(0, len(lens), q, k, v, b.pages, _dev(lens), rope=rope)
    assert torch.equal(a.k.view(torch.int16), b.k.view(torch.int16)) and torch.equal(a.v.view(torch.int16), b.v.view(torch.int16))
    for r in rigs:
        for i, n in enumerate(lens):
            if n:
                r.rows[i] = [pool.view(-1, Hkv, 128)[r.slots(i, r.keep[i])] for pool in (r.k, r.v)]
        assert r.plan.flux_plan_status() == 0
    a.check(qr, want)
    if rope:
        b.check(*_with_mag(got, *paged.turned(_f64(q), [max(n - 1, 0) for n in lens], _inv_freq(rot), None if w[0] is None else _f64(w[0]), pairs=pairs)))
    else:
        b.check(qr, got)


@pytest.mark.parametrize("Hq,Hkv,ctx,page", [(32, 8, [20000], 16), (28, 4, [131, 30001, 4], 64), (16, 1, [40000, 1], 128), (36, 3, [12345] * 3, 32), (8, 2, list(range(1, 301)), 16)])
def test_step_split_over_many_ctas(flux, Hq, Hkv, ctx, page):
    modes = [(i + 1) % 2 for i in range(len(ctx))]
    r = Rig(flux, Hq, Hkv, 128, 2048, modes, ctx, page, seed=sum(ctx) % 1000)
    x = _rows(r.gen, len(ctx), Hq + 2 * Hkv)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    rope = flux.Rope(_inv_freq(128, 5e5), device=DEV)
    at = [n - 1 for n in ctx]
    want = r.plan.flux_qk_norm_rope(rope, None, k, _dev(at))[1]
    out = r.plan.flux_attn_decode_step_paged(0, len(ctx), q, k, v, r.pages, _dev(ctx), rope=rope)
    again = r.plan.flux_attn_decode_step_paged(0, len(ctx), q, k, v, r.pages, _dev(ctx), rope=rope)
    assert torch.equal(out, again)
    for b, n in enumerate(ctx):
        assert torch.equal(r.k.view(-1, Hkv, 128)[r.slots(b, [n - 1])][0], want[b]) and torch.equal(r.v.view(-1, Hkv, 128)[r.slots(b, [n - 1])][0], v[b])
        r.rows[b] = [pool.view(-1, Hkv, 128)[r.slots(b, r.keep[b])] for pool in (r.k, r.v)]
    yq, mag = paged.turned(_f64(q), at, _inv_freq(128, 5e5))
    r.check(yq, out, "step", mag)
    assert r.plan.flux_plan_status() == 0


def _with_mag(out, q, mag):
    return q, out, "step", mag


@pytest.mark.parametrize("page", [16, 64])
def test_steps_right_behind_one_another_with_overlap(flux, page):
    """One layer, token after token, nothing between the launches: each reads what the one before has stored."""
    lens, steps = [1, 15, 30, 700, 3000], 40
    found = []
    for overlap in (False, True):
        r = Rig(flux, 8, 2, 20, 100, [1, 0, 1, 0, 1], lens, page, seed=2, room=steps + 1)
        table = r.table.clone()
        n = 0
        for b in range(len(lens)):                            # pages for what is to come
            for j in range(lens[b] // page, (lens[b] + steps) // page + 1):
                if table[b, j] < 0:
                    table[b, j] = r.n_pages + n
                    n += 1
        k, v = (torch.cat([x, torch.zeros(n, page, 2, 128, dtype=torch.bfloat16, device=DEV)]) for x in (r.k, r.v))
        pages = flux.Pages(k, v, table)
        rope = flux.Rope(_inv_freq(128), device=DEV)
        x = [_rows(r.gen, len(lens), 12) for _ in range(steps)]
        at = [_dev([m + i + 1 for m in lens]) for i in range(steps)]
        outs = [torch.empty(len(lens), 8, 128, dtype=torch.bfloat16, device=DEV) for _ in range(steps)]
        r.plan.flux_plan_set_launch_overlap(overlap)
        torch.cuda.synchronize()
        for i in range(steps):
            r.plan.flux_attn_decode_step_paged(0, len(lens), x[i][:, :8], x[i][:, 8:10], x[i][:, 10:], pages, at[i], rope=rope, out=outs[i])
        assert r.plan.flux_plan_status() == 0
        found.append([torch.stack(outs), k.view(torch.int16), v.view(torch.int16)])
    assert all(torch.equal(a, b) for a, b in zip(*found))


def test_step_without_its_page_loses_the_token(flux):
    r = Rig(flux, 8, 2, 4, 8, [1, 1], [40, 17], 16)
    r.table[1, 1] = -1
    x = _rows(r.gen, 2, 12)
    before = r.k.clone()
    out = r.plan.flux_attn_decode_step_paged(0, 2, x[:, :8], x[:, 8:10], x[:, 10:], r.pages, _dev(r.ctx))
    assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE
    _check_decode(_f64(x[1, :8]), _f64(r.rows[1][0][:16]), _f64(r.rows[1][1][:16]), _f64(out[1]))
    before.view(-1, 2, 128)[r.slots(0, [39])] = x[:1, 8:10]
    assert torch.equal(r.k.view(torch.int16), before.view(torch.int16))


# ---- bookkeeping -----------------------------------------------------------------------------------------------------

class Book:
    """A pool on the device beside the oracle's."""

    def __init__(self, flux, n_pages, rows, cols, page, Hkv=1, slabs=2, seed=0):
        self.flux, self.plan = flux, _plan(flux, Hkv, Hkv)
        gen = _gen(seed)
        self.data = torch.randint(-30000, 30000, (slabs, n_pages, page, Hkv * 128), generator=gen, device=DEV, dtype=torch.int16)
        self.table = torch.full((rows, cols), -1, dtype=torch.int32, device=DEV)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
        self.pool = flux.PagePool(self.table, self.refs, [x.view(torch.bfloat16).view(n_pages, page, Hkv, 128) for x in self.data])
        self.page = page
        self.copy()

    def copy(self):
        self.o = paged.Pool(self.table.cpu().numpy(), self.refs.cpu().numpy(), self.data.cpu().numpy(), self.page)

    def same(self, what=""):
        f = self.flux
        bits = self.plan.flux_plan_status(raise_on_flag=False)
        want = (f.FLUX_STATUS_BAD_PAGE if self.o.bad_page else 0) | (f.FLUX_STATUS_BAD_LENGTH if self.o.bad_length else 0) | (f.FLUX_STATUS_NO_PAGES if self.o.no_pages else 0)
        self.o.bad_page = self.o.bad_length = self.o.no_pages = False
        assert bits == want, (what, bits, want)
        assert np.array_equal(self.table.cpu().numpy(), self.o.table), what
        assert np.array_equal(self.refs.cpu().numpy(), self.o.refs), what
        assert np.array_equal(self.data.cpu().numpy(), self.o.data), what

    def reserve(self, rows, a, b):
        got = self.plan.flux_pages_reserve(self.pool, None if rows is None else _dev(rows), _dev(a), _dev(b))
        want = self.o.reserve(list(range(len(a))) if rows is None else rows, a, b)
        assert got.tolist() == want
        self.same("reserve")
        return want

    def fork(self, src, dst, n):
        self.plan.flux_pages_fork(self.pool, _dev(src), _dev(dst), _dev(n))
        self.o.fork(src, dst, n)
        self.same("fork")

    def release(self, rows, a, b):
        self.plan.flux_pages_release(self.pool, _dev(rows), _dev(a), _dev(b))
        self.o.release(rows, a, b)
        self.same("release")

    def compact(self):
        to, used = self.plan.flux_pages_compact(self.pool)
        want, n = self.o.compact()
        assert np.array_equal(to.cpu().numpy(), want) and int(used) == n
        self.same("compact")


@pytest.mark.parametrize("n_pages,rows,cols,page,slabs,seed", [(60, 6, 9, 16, 2, 1), (1024, 20, 40, 16, 1, 2), (1500, 33, 65, 32, 3, 3), (5000, 100, 70, 16, 2, 4), (2100, 8, 300, 64, 1, 5), (90, 12, 8, 128, 4, 6),
                                                                (70, 9, 5, 256, 2, 7)])
def test_random_bookkeeping(flux, n_pages, rows, cols, page, slabs, seed):
    p = Book(flux, n_pages, rows, cols, page, slabs=slabs, seed=seed)
    rng = np.random.default_rng(seed)
    lens = [0] * rows
    for turn in range(60):
        some = [int(x) for x in rng.permutation(rows)[:int(rng.integers(1, rows + 1))]]
        what = rng.choice(["grow", "token", "token", "fork", "drop", "middle", "cut", "compact"])
        if what in ("grow", "token"):
            new = [min(cols * page, lens[r] + (1 if what == "token" else int(rng.integers(0, cols * page // 3)))) for r in some]
            for r, n, ok in zip(some, new, p.reserve(some, [lens[r] for r in some], new)):
                lens[r] = n if ok else lens[r]
        elif what == "fork":
            src = [int(rng.integers(0, rows)) for _ in some]
            n = [int(rng.integers(0, lens[s] + 1)) if rng.random() < 0.3 else lens[s] for s in src]
            p.fork(src, some, n)
            before = dict(zip(some, n))
            lens = [before.get(r, x) for r, x in enumerate(lens)]
        elif what == "drop":
            some = some[:max(len(some) // 3, 1)]
            p.release(some, [0] * len(some), [2 ** 31 - 1] * len(some))
            lens = [0 if r in some else x for r, x in enumerate(lens)]
        elif what == "middle":
            p.release(some, [int(rng.integers(0, 50))] * len(some), [max(lens[r] - int(rng.integers(0, 100)), 0) for r in some])
        elif what == "cut":
            lens = [int(rng.integers(0, x + 1)) if r in some else x for r, x in enumerate(lens)]
            p.release(some, [lens[r] for r in some], [2 ** 31 - 1] * len(some))
        else:
            p.compact()
    held = p.o.table[p.o.table >= 0]
    assert np.array_equal(np.bincount(held, minlength=n_pages), p.o.refs)


def test_beams_of_a_group_write_on(flux):
    """All holders of a begun page are listed: the last keeps it; with one that is not listed everybody copies; len at a page's end copies nothing."""
    p = Book(flux, 300, 40, 8, 16, Hkv=2)
    p.reserve([0, 8], [0, 0], [37, 32])
    p.fork([0] * 7 + [8] * 4, list(range(1, 8)) + list(range(9, 13)), [37] * 7 + [32] * 4)
    p.reserve(list(range(8)), [37] * 8, [38] * 8)
    p.reserve([8, 9, 10, 11, 12], [32] * 5, [33] * 5)
    p.fork([0, 0, 8], [20, 21, 22], [38, 38, 33])
    p.reserve([21, 0], [38, 38], [39, 40])                    # row 20 holds it too
    p.reserve([20], [38], [39])
    p.reserve([22], [20], [21])                               # a begun page below the sharing one
    p.reserve(None, [38] * 8, [38] * 8)                       # nothing to do
    assert p.plan.flux_pages_reserve(p.pool, _dev([]), _dev([]), _dev([])).numel() == 0


@pytest.mark.parametrize("n", [1025, 4096])
def test_many_rows_at_once(flux, n):
    p = Book(flux, 3 * n + 100, n, 6, 16, slabs=1)
    order = [int(x) for x in np.random.default_rng(n).permutation(n)]
    p.reserve(order, [0] * n, [(r % 3) * 16 + 5 for r in order])
    lens = [(r % 3) * 16 + 5 for r in range(n)]
    src = [r - r % 12 + (r % 4) for r in range(n - n % 12)]
    p.fork(src, list(range(len(src))), [lens[s] for s in src])
    lens[:len(src)] = [lens[s] for s in src]
    p.reserve(order, [lens[r] for r in order], [lens[r] + 1 for r in order])
    p.release(order[: n // 2], [0] * (n // 2), [2 ** 31 - 1] * (n // 2))
    p.compact()


def test_wide_tables_and_large_pools(flux):
    """Rows of thousands of pages, and a pool of more chunks than a CTA has threads."""
    p = Book(flux, 300 * 1024 + 77, 3, 9000, 16, slabs=1, seed=9)
    p.reserve([2, 0], [0, 0], [9000 * 16, 7000 * 16 + 3])
    p.release([2], [100], [8000 * 16])
    p.fork([0], [1], [5000 * 16 + 7])
    p.reserve([1, 2], [5000 * 16 + 7, 50], [8000 * 16, 200 * 16])
    p.compact()
    p.release([0, 1, 2], [0] * 3, [2 ** 31 - 1] * 3)
    assert int(p.refs.sum()) == 0
    p.compact()


def test_rows_that_ask_for_more_than_32_bits_count(flux):
    """33 rows of 2^26 pages: together beyond 2^31, so none of them is served, and the one before them is."""
    n, cols, n_pages = 34, 1 << 26, 40
    table = torch.full((n, cols), -1, dtype=torch.int32, device=DEV)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    plan = _plan(flux, 1, 1)
    pool = flux.PagePool(table, refs, [torch.zeros((n_pages, 16, 1, 128), dtype=torch.bfloat16, device=DEV)])
    granted = plan.flux_pages_reserve(pool, None, _dev([0] * n), _dev([48] + [1 << 30] * (n - 1)))
    assert plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_NO_PAGES
    assert granted.tolist() == [1] + [0] * (n - 1) and table[0, :4].tolist() == [0, 1, 2, -1] and refs.sum().item() == 3
    assert all(int((row != -1).sum()) == (3 if i == 0 else 0) for i, row in enumerate(table))


def test_bookkeeping_refusals(flux):
    p = Book(flux, 50, 5, 6, 16)
    p.reserve([0, 1, 2], [0, 0, 0], [40, 20, 90])
    p.reserve([0, 5, -1, 1, 0], [40, 0, 0, 20, 40], [60, 5, 5, 30, 80])          # rows outside the table, a row twice
    p.reserve([0, 1, 2, 3], [-1, 20, 96, 0], [5, 19, 97, 2 ** 31 - 1])           # lengths that cannot be
    p.fork([0, 0, 7, 1, 0], [3, 3, 4, 9, -2], [30, 30, 10, 10, 10])
    p.fork([0, 1], [3, 4], [-1, 97])
    p.release([9, -1, 1], [0, 0, -4], [90, 90, 90])
    p.release([1, 1, 1], [0, 0, 0], [90, 90, 90])                                # the same row again: nothing is left
    # entries that cannot be
    for entry in (50, -2, 2 ** 31 - 1, 49):                                      # page 49 is free
        p.table[4, 1] = entry
        p.copy()
        p.reserve([4, 2], [20, 90], [25, 91])
        p.table[4, 1] = -1
        p.copy()
    p.table[4, 1], p.table[4, 2] = 49, 77
    p.copy()
    p.plan.flux_pages_compact(p.pool)
    assert p.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE and (p.table[4] == -1).all()
    p.copy()
    # a page that nobody counted is given up
    p.table[4, 0] = 49
    p.plan.flux_pages_release(p.pool, _dev([4]), _dev([0]), _dev([90]))
    assert p.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_PAGE and int(p.refs[49]) == 0 and int(p.table[4, 0]) == -1
    one = _dev([0])
    for call, code in ((lambda: p.plan.flux_pages_reserve(p.pool, None, _dev([0] * 6), _dev([0] * 6)), flux.FLUX_E_INVALID_ARG),
                       (lambda: p.plan.flux_pages_release(p.pool, _dev([0] * 4097), _dev([0] * 4097), _dev([0] * 4097)), flux.FLUX_E_CAPACITY)):
        with pytest.raises(flux.FluxError) as e:
            call()
        assert e.value.code == code
    other = _plan(flux, 2, 2)
    for call in (lambda: other.flux_pages_compact(p.pool), lambda: p.plan.flux_pages_release(p.pool, one, one.long(), one), lambda: p.plan.flux_pages_fork(p.pool, one, one.cpu(), one),
                 lambda: p.plan.flux_pages_fork(p.pool, one, _dev([]), one)):
        with pytest.raises(ValueError):
            call()


# ---- together --------------------------------------------------------------------------------------------------------

def _serve(flux, graph, overlap):
    """Prompts through norm, rotation, packed prefill and store; beams forked; decode steps whose lengths advance on the device; a request
    released, the pool compacted, steps again.  Returns every output, and checks each against the oracle over the rows that were stored."""
    Hq, Hkv, S, W, page, modes, n_pages = 8, 2, 20, 60, 16, [1, 1, 0, 1], 64
    B = len(modes)
    plan = _plan(flux, Hq, Hkv, S, W, modes, 400)
    gen = _gen(11)
    w = [torch.rand(128, generator=gen, device=DEV).bfloat16() for _ in "qk"]
    rope = flux.Rope(_inv_freq(128), q_weight=w[0], k_weight=w[1], device=DEV)
    k, v = (torch.full((n_pages, page, Hkv, 128), NAN, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    table, refs = torch.full((B, 25), -1, dtype=torch.int32, device=DEV), torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    pages, pool = flux.Pages(k, v, table), flux.PagePool(table, refs, [k, v])
    new = [150, 0, 230, 33]
    lens = _dev(new)
    plan.flux_pages_reserve(pool, None, _dev([0] * B), lens)
    x = _rows(gen, sum(new), Hq + 2 * Hkv)
    kr = torch.empty(sum(new), Hkv, 128, dtype=torch.bfloat16, device=DEV)
    q = plan.flux_paged_store(pages, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], _dev(_cum(new)), _dev([0] * B), rope=rope, q=x[:, :Hq], k_out=kr)
    prompt = plan.flux_attn_prefill_packed(0, q, kr, x[:, Hq + Hkv:], np.array(_cum(new), dtype=np.int32))
    hist = [[t[a:e] for t in (kr, x[:, Hq + Hkv:])] for a, e in zip(_cum(new), _cum(new)[1:])]
    for b, n in enumerate(new):                               # the last row of every prompt
        if n:
            keep = kvq.kept(n, modes[b] == 1, S, W)
            ref, A, _, _ = kvq.attend(_f64(q[_cum(new)[b + 1] - 1]), _f64(hist[b][0][keep]), _f64(hist[b][1][keep]), 1 / np.sqrt(128))
            # output and weights in bf16, weights rounded in the numerator alone; the rest as in a decode
            assert (np.abs(_f64(prompt[_cum(new)[b + 1] - 1]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -7 * A).all()
    plan.flux_pages_fork(pool, _dev([0]), _dev([1]), _dev([150]))
    new[1], hist[1] = 150, list(hist[0])
    lens = _dev(new)
    fused, out = torch.empty(B, Hq + 2 * Hkv, 128, dtype=torch.bfloat16, device=DEV), torch.empty(B, Hq, 128, dtype=torch.bfloat16, device=DEV)
    nxt, sink, edge = lens.clone(), _dev([S]), torch.zeros(1, dtype=torch.int32, device=DEV)
    sparse = _dev([2])

    def step():
        torch.add(lens, 1, out=nxt)
        plan.flux_pages_reserve(pool, None, lens, nxt)
        torch.sub(nxt[2:3], W, out=edge)
        plan.flux_pages_release(pool, sparse, sink, edge)     # what the sparse request's step does not need any more
        torch.mul(fused, 1, out=fused)                        # (a kernel of the program's between the tables and the decode)
        plan.flux_attn_decode_step_paged(0, B, fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:], pages, nxt, rope=rope, out=out)
        lens.copy_(nxt)

    plan.flux_plan_set_launch_overlap(overlap)
    run = step
    if graph:
        fused.zero_()
        keep = [t.clone() for t in (k, v, table, refs, lens)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for t, s in zip((k, v, table, refs, lens), keep):
            t.copy_(s)
        run = g.replay
    found = []
    for i in range(24):
        y = _rows(gen, B, Hq + 2 * Hkv)
        fused.copy_(y)
        run()
        at = [n + i for n in new]
        _, yk = plan.flux_qk_norm_rope(rope, None, y[:, Hq:Hq + Hkv], _dev(at))
        yq, mag = paged.turned(_f64(y[:, :Hq]), at, _inv_freq(128), _f64(w[0]))
        found.append(out.clone())
        for b in range(B):
            hist[b] = [torch.cat([h, t[b:b + 1]]) for h, t in zip(hist[b], (yk, y[:, Hq + Hkv:]))]
            keep = kvq.kept(at[b] + 1, modes[b] == 1, S, W)
            _check_decode(yq[b], _f64(hist[b][0][keep]), _f64(hist[b][1][keep]), _f64(out[b]), "step %d request %d" % (i, b), mag[b])
        if i == 11:
            plan.flux_pages_release(pool, _dev([3]), _dev([0]), _dev([2 ** 31 - 1]))
            n = at[0] + 1
            plan.flux_pages_fork(pool, _dev([0]), _dev([3]), _dev([n]))             # a third beam of the first prompt
            new[3] = n - (i + 1)
            hist[3] = list(hist[0])
            lens[3] = n
            plan.flux_pages_compact(pool)
            used = int((refs > 0).sum())
            assert (refs[:used] > 0).all() and (refs[used:] == 0).all()
    assert plan.flux_plan_status() == 0
    assert torch.equal(torch.bincount(table[table >= 0].long(), minlength=n_pages).int(), refs)
    assert int((table[2] >= 0).sum()) <= 2 + 5                # sink and window, no more
    return torch.stack(found)


def test_calls_together_as_a_server_makes_them(flux):
    want = _serve(flux, False, False)
    assert torch.equal(_serve(flux, True, False), want)       # steps replayed from one captured graph
    assert torch.equal(_serve(flux, True, True), want)


def test_another_stream(flux):
    r = Rig(flux, 8, 2, 20, 100, [1, 0, 1], [900, 4000, 77], 32)
    q = _rows(r.gen, 3, 8)
    want = r.decode(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        big = torch.randn(4000, 4000, device=DEV)
        for _ in range(5):
            big = big @ big * 1e-4
        late = torch.where(big.sum().isnan(), q, q)           # ready only when the products are
        got = r.decode(late)
    side.synchronize()
    assert torch.equal(got, want) and r.plan.flux_plan_status() == 0
