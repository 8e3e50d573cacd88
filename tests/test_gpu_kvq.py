"""GPU parity of the 8-bit KV cache (store, load) and of the decode that reads it, against the fp64 oracle.

What a cache holds is compared exactly: a loaded entry is code x scale in fp32 rounded to bf16 -- for e4m3 the value itself (four
significant bits times a power of two), for int8 the fp64 value rounded to fp32 and then to bf16.

Decode outputs: with p_j the softmax weights and A = sum_j p_j |v_j|, an element is off by at most
    2^-8 |ref|                  bf16 output (half a step)
  + 2^-11 A                     weights rounded to fp16 (tail keys: to bf16, 2^-8 of their part of A)
  + 2^-34 M sum_j |v_j| / s_j   (keys in 8 bits) with s_j the scale of key j's block and M = max_j p_j s_j.  The kernel's weight of the codes
                                is w_j = p_j s_j up to a common factor that brings the largest into 2^10 .. 2^14; in fp16, w_j below 2^-14 is
                                off by half of 2^-24 -- absolutely, so by 2^-35 of the largest w -- and multiplies |v_j| / s_j
  + 2 D A                       weights off by a factor 1 + D in numerator and row sum: D = 2^-20 (log2, ex2, reciprocal, fp32 sums and rescaling by
                                at most a few dozen factors of 2^-24 each) + the error of a score, 2^-16 of the largest
                                sum_d |q_d k_d| (128 fp32 additions, in any order and rounded or cut off, of products of exact operands;
                                query entries below 2^-14 of their row's largest are off by 2^-25 of it, less than that again)
"""
import numpy as np
import pytest
import torch

from oracle import kvq
from paper_2604_07394_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FMTS = ["e4m3", "int8"]


@pytest.fixture(scope="module")
def flux():
    from paper_2604_07394_b200 import build, flux as f
    build.build()
    f.load()
    return f


def _fmt(flux, fmt):
    return {"e4m3": flux.FLUX_KVQ_E4M3, "int8": flux.FLUX_KVQ_INT8}[fmt]


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cum(x):
    return [0] + np.cumsum(x).tolist()


class Rig:
    """A plan of one layer, guarded cache buffers for every request, and the bf16 history the caches were given."""
    GUARD = 256

    def __init__(self, flux, fmt, Hq, Hkv, S, W, modes, max_ctx, layout=0, seed=1):
        self.flux, self.fmt, self.f, self.S, self.W, self.modes, self.Hq, self.Hkv = flux, fmt, _fmt(flux, fmt), S, W, modes, Hq, Hkv
        self.B = len(modes)
        self.plan = flux.Plan(flux.make_config(1, Hq, Hkv, S, W, self.B, max_ctx, kv_layout=layout), DEV)
        self.plan.flux_router_apply(mask=np.array([[m] for m in modes], dtype=np.uint8))
        self.size = [flux.flux_kvq_cache_size(self.plan.cfg, layout == 1 and m == 0, max_ctx) for m in modes]
        # 0xff: NaN codes, NaN scales and NaN rows wherever nothing has been stored
        self.bufs = [[torch.full((s + 2 * self.GUARD,), 0xff, dtype=torch.uint8, device=DEV) for s in self.size] for _ in "kv"]
        self.kt, self.vt = (flux.pointer_table([x[self.GUARD:] for x in b], DEV) for b in self.bufs)
        self.hist = [[torch.zeros(0, Hkv, 128, dtype=torch.bfloat16, device=DEV) for _ in modes] for _ in "kv"]
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(seed)

    def rows(self, n, heads=None):
        x = torch.randn(n, heads or self.Hkv, 128, generator=self.gen, device=DEV)
        big = torch.ones(128, device=DEV)
        big[5::31] = 6.0                       # a few large channels, as keys have
        return (x * big).to(torch.bfloat16)

    def store(self, lens, k=None, v=None):
        k = self.rows(sum(lens)) if k is None else k
        v = self.rows(sum(lens)) if v is None else v
        pos = [len(h) for h in self.hist[0]]
        self.plan.flux_kvq_store(0, self.f, k, v, _dev(_cum(lens)), _dev(pos), self.kt, self.vt)
        for h, x in zip(self.hist, (k, v)):
            for b, (a, e) in enumerate(zip(_cum(lens), _cum(lens)[1:])):
                h[b] = torch.cat([h[b], x[a:e]])

    @property
    def ctx(self):
        return [len(h) for h in self.hist[0]]

    def load(self, pos, lens, ctx=None):
        return self.plan.flux_kvq_load(0, self.f, self.kt, self.vt, _dev(ctx or self.ctx), _dev(_cum(lens)), _dev(pos), sum(lens))

    def values(self, b):
        return [kvq.cache_values(h[b].double().cpu().numpy(), self.fmt) for h in self.hist]

    def guards(self):
        return all(bool((x[:self.GUARD] == 0xff).all()) and bool((x[-self.GUARD:] == 0xff).all()) for b in self.bufs for x in b)

    def decode(self, q=None, step=None):
        q = self.rows(self.B, self.Hq) if q is None else q
        ctx = _dev(self.ctx)
        if step is None:
            return q, self.plan.flux_attn_decode_kvq(0, self.B, self.f, q, self.kt, self.vt, ctx)
        return q, self.plan.flux_attn_decode_step_kvq(0, self.B, self.f, q, step[0], step[1], self.kt, self.vt, ctx)

    def check(self, q, out, what=""):
        sc = 1 / np.sqrt(128)
        for b in range(self.B):
            n = self.ctx[b]
            got = out[b].double().cpu().numpy()
            if n == 0:
                assert (got == 0).all(), what
                continue
            k, v = self.values(b)
            keep = kvq.kept(n, self.modes[b] == 1, self.S, self.W)
            ref, A, mag, p = kvq.attend(q[b].double().cpu().numpy(), k[keep], v[keep], sc)
            tail = keep >= n // 16 * 16
            At = np.einsum("hm,mhd->hd", p[:, tail], np.abs(np.repeat(v[keep][tail], self.Hq // self.Hkv, axis=1)))
            s = np.repeat(kvq.key_scales(self.hist[1][b].double().cpu().numpy(), self.fmt)[keep], self.Hq // self.Hkv, axis=1)   # [m][Hq]
            vr = np.abs(np.repeat(v[keep], self.Hq // self.Hkv, axis=1)) / np.where(s > 0, s, np.inf)[:, :, None]
            under = 2.0 ** -34 * (p * s.T).max(1)[:, None] * vr.sum(0)
            d = 2.0 ** -20 + 2.0 ** -16 * mag[:, None]
            tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -11 * A + 2.0 ** -8 * At + 2 * d * A + under
            err = np.abs(got - ref)
            ok = bool(np.isfinite(got).all()) and bool((err <= tol).all())
            assert ok, "%s request %d: %.3e over tolerance, at most %.2f of it" % (
                what, b, (err - tol).max(), (err / tol).max())


def _as_loaded(values):
    return torch.from_numpy(values.astype(np.float32)).to(torch.bfloat16)


# ---- store and load ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("Hkv", [1, 2, 5, 8])
def test_store_then_load_every_length(flux, fmt, Hkv):
    lens = [0, 1, 15, 16, 17, 31, 32, 0, 63, 64, 65, 130, 257, 0]
    r = Rig(flux, fmt, Hkv, Hkv, 4, 8, [1] * len(lens), 300)
    r.store(lens)
    k, v = r.load([0] * len(lens), lens)
    for b, (a, e) in enumerate(zip(_cum(lens), _cum(lens)[1:])):
        for got, want in zip((k[a:e], v[a:e]), r.values(b)):
            assert torch.equal(got.cpu(), _as_loaded(want)), (b, lens[b])
    assert r.guards() and r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_cache_does_not_depend_on_how_rows_arrive(flux, fmt):
    total = [100, 37, 16, 150]
    r = Rig(flux, fmt, 4, 2, 4, 8, [1] * 4, 200)
    k, v = r.rows(sum(total)), r.rows(sum(total))
    r.store(total, k, v)
    want = r.load([0] * 4, total)
    rng = np.random.default_rng(3)
    for trial in range(3):
        s = Rig(flux, fmt, 4, 2, 4, 8, [1] * 4, 200)
        done = [0] * 4
        while done != total:
            lens = [min(t - d, int(rng.choice([0, 1, 1, 3, 15, 16, 17, 40]))) for t, d in zip(total, done)]
            idx = sum((list(range(a + d, a + d + n)) for a, d, n in zip(_cum(total), done, lens)), [])
            s.store(lens, k[idx], v[idx])
            done = [d + n for d, n in zip(done, lens)]
        got = s.load([0] * 4, total)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and s.guards()
        assert s.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_load_ranges_leave_other_rows(flux, fmt):
    r = Rig(flux, fmt, 4, 2, 4, 8, [1] * 3, 200)
    r.store([100, 50, 33])
    pos, lens = [17, 0, 32], [70, 0, 1]
    k = torch.full((90, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    r.plan.flux_kvq_load(0, r.f, r.kt, r.vt, _dev(r.ctx), _dev([3, 73, 73, 74]), _dev(pos), 90, k, v)
    for got, b0, b2 in zip((k, v), r.values(0), r.values(2)):
        assert torch.equal(got[3:73].cpu(), _as_loaded(b0[17:87])) and torch.equal(got[73:74].cpu(), _as_loaded(b2[32:33]))
        assert bool((got[:3] == 7).all()) and bool((got[74:] == 7).all())
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_store_extreme_and_non_finite_values(flux, fmt):
    r = Rig(flux, fmt, 2, 2, 4, 8, [1], 200)
    k, v = r.rows(96), r.rows(96)
    k[0:16, 0] = 0.0
    k[16:32, 0] *= 2.0 ** -120
    k[32:48, 0] = 3.3895313892515355e38
    k[33:48, 0, ::2] = -1.0e36
    k[48:64, 0] *= torch.exp2(torch.randint(-30, 30, (16, 128), generator=r.gen, device=DEV).float()).to(torch.bfloat16)
    v[0:16, 1, :] = torch.arange(-64, 64, device=DEV).to(torch.bfloat16) + 0.5      # int8 with amax 127: codes halfway between integers
    v[0, 1, 0] = 127.0
    r.store([96], k, v)
    for got, want in zip(r.load([0], [96]), r.values(0)):
        assert torch.equal(got.cpu(), _as_loaded(want))
    assert r.plan.flux_plan_status() == 0
    k = r.rows(21)
    v = r.rows(21)
    k[3, 0, 5], k[4, 1, 127], v[7, 0, 0], v[20, 1, 3] = float("nan"), float("inf"), -float("inf"), float("nan")
    r2 = Rig(flux, fmt, 2, 2, 4, 8, [1], 200)
    r2.store([21], k, v)
    assert r2.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_NONFINITE
    for got, want in zip(r2.load([0], [21]), r2.values(0)):
        assert torch.equal(got.cpu(), _as_loaded(want))


@pytest.mark.parametrize("fmt", FMTS)
def test_store_of_strided_rows(flux, fmt):
    r = Rig(flux, fmt, 8, 2, 4, 8, [1, 1], 200)
    fused = r.rows(70, 12)                       # a projection output [q heads | k heads | v heads]
    k, v = fused[:, 8:10], fused[:, 10:12]
    r.store([40, 30], k, v)
    got = r.load([0, 0], [40, 30])
    s = Rig(flux, fmt, 8, 2, 4, 8, [1, 1], 200)
    s.store([40, 30], k.contiguous(), v.contiguous())
    want = s.load([0, 0], [40, 30])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("S,W", [(0, 1), (5, 33), (64, 64), (70, 130)])
@pytest.mark.parametrize("fmt", FMTS)
def test_compact_cache_keeps_sink_and_window(flux, fmt, S, W):
    r = Rig(flux, fmt, 2, 2, S, W, [0, 1], 700, layout=1)
    rng = np.random.default_rng(S + W)
    for n in (300, 5, 1, 1, 1, 60, 16, 17, 120, 1, 2):
        r.store([n, int(rng.integers(0, 30))])
        n0 = r.ctx[0]
        k, v = r.load([0, 0], r.ctx)
        held = kvq.kept(n0, False, S, W)
        for got, want in zip((k, v), r.values(0)):
            got = got[:n0].cpu()
            want = _as_loaded(want)
            assert torch.equal(got[held], want[held]), (n, n0)
            rest = np.setdiff1d(np.arange(n0), held)       # what has been dropped reads as zero (a block may still be held)
            assert bool(((got[rest] == want[rest]) | (got[rest] == 0)).all())
    assert r.guards() and r.plan.flux_plan_status() == 0


def test_begun_block_may_be_stored_again(flux):
    r = Rig(flux, "int8", 2, 2, 4, 8, [1, 1], 100)
    r.store([47, 20])
    k, v = r.rows(2), r.rows(2)
    want = None
    for _ in range(3):                           # position 47 completes its block, position 20 does not
        r.plan.flux_kvq_store(0, r.f, k, v, _dev([0, 1, 2]), _dev([47, 20]), r.kt, r.vt)
        got = r.load([0, 0], [48, 21], ctx=[48, 21])
        want = want or got
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(want[0][68].cpu(), k[1].cpu()) and r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("first", [32, 21])
def test_complete_newest_block_may_be_stored_again_in_part(flux, first):
    """A call of several blocks that ends on a block's last position, then that block's last tokens once more."""
    for fmt in FMTS:
        r = Rig(flux, fmt, 2, 2, 4, 8, [1, 1], 100)
        r.store([0, 5])
        r.store([first, 27])                     # request 1 begins inside a block and ends with position 31
        r.store([-first % 48 if first % 16 else 0, 0])
        want = r.load([0, 0], r.ctx)
        n = r.ctx
        for back in (1, 6):
            k, v = (torch.cat([h[0][n[0] - back:], h[1][n[1] - back:]]) for h in r.hist)
            r.plan.flux_kvq_store(0, r.f, k, v, _dev([0, back, 2 * back]), _dev([n[0] - back, n[1] - back]), r.kt, r.vt)
            got = r.load([0, 0], n)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (fmt, back)
        q = r.rows(2)
        out = r.plan.flux_attn_decode_step_kvq(0, 2, r.f, q, *(torch.stack([h[0][-1], h[1][-1]]) for h in r.hist), r.kt, r.vt, _dev(n))
        r.check(q, out)
        got = r.load([0, 0], n)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and r.plan.flux_plan_status() == 0


def test_one_lost_cache_and_wild_lengths_leave_the_request_alone(flux):
    r = Rig(flux, "e4m3", 4, 2, 4, 8, [1, 1], 100)
    r.store([30, 20])
    before = [x.clone() for b in r.bufs for x in b]
    k, v = r.rows(9), r.rows(9)
    half = r.vt.clone()
    half[0] = 0
    rows, pos = _dev([0, 5, 5]), _dev([30, 20])
    for kt, vt in ((r.kt, half), (half, r.vt)):
        r.plan.flux_kvq_store(0, r.f, k, v, rows, pos, kt, vt)
        assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_POINTER
        assert all(torch.equal(x, y) for x, y in zip(before, (x for b in r.bufs for x in b)))
    for ctx in ([-2 ** 31, 20], [-1, 20], [4, 20], [101, 20]):
        out = r.plan.flux_kvq_load(0, r.f, r.kt, r.vt, _dev(ctx), rows, _dev([0, 0]), 5)
        assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_LENGTH, ctx


def test_store_and_load_refusals(flux):
    r = Rig(flux, "e4m3", 4, 2, 4, 8, [1, 1], 100)
    r.store([30, 20])
    before = [x.clone() for b in r.bufs for x in b]
    k, v = r.rows(90), r.rows(90)

    def flagged(call, bits):
        call()
        assert r.plan.flux_plan_status(raise_on_flag=False) == bits
        assert all(torch.equal(x, y) for x, y in zip(before, (x for b in r.bufs for x in b)))

    bad = flux.FLUX_STATUS_BAD_LENGTH
    st = lambda rows, pos: (lambda: r.plan.flux_kvq_store(0, r.f, k, v, _dev(rows), _dev(pos), r.kt, r.vt))  # noqa: E731
    flagged(st([0, 90, 90], [30, 20]), bad)          # past max_context
    flagged(st([0, 0, 91], [30, 20]), bad)           # past the rows given
    flagged(st([10, 5, 5], [30, 20]), bad)           # rows run backwards
    flagged(st([0, 1, 1], [-1, 20]), bad)
    flagged(st([-3, 0, 0], [30, 20]), bad)
    null = torch.zeros(2, dtype=torch.int64, device=DEV)
    odd = r.kt + 4
    for table in (null, odd):
        flagged(lambda: r.plan.flux_kvq_store(0, r.f, k, v, _dev([0, 1, 2]), _dev([30, 20]), table, table), flux.FLUX_STATUS_BAD_POINTER)
        flagged(lambda: r.plan.flux_kvq_load(0, r.f, table, table, _dev([30, 20]), _dev([0, 1, 2]), _dev([0, 0]), 2), flux.FLUX_STATUS_BAD_POINTER)
        flagged(lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(2, 4), table, table, _dev([30, 20])), flux.FLUX_STATUS_BAD_POINTER)
    flagged(lambda: r.plan.flux_kvq_load(0, r.f, r.kt, r.vt, _dev([30, 20]), _dev([0, 31, 31]), _dev([0, 0]), 31), bad)
    flagged(lambda: r.plan.flux_kvq_load(0, r.f, r.kt, r.vt, _dev([30, 20]), _dev([0, 3, 3]), _dev([28, 0]), 31), bad)
    for call, code in (
            (lambda: r.plan.flux_kvq_store(1, r.f, k, v, _dev([0, 1, 2]), _dev([30, 20]), r.kt, r.vt), flux.FLUX_E_INVALID_ARG),
            (lambda: r.plan.flux_kvq_store(0, 2, k, v, _dev([0, 1, 2]), _dev([30, 20]), r.kt, r.vt), flux.FLUX_E_INVALID_ARG),
            (lambda: r.plan.flux_kvq_store(0, r.f, k, v, _dev([0, 1, 2, 3]), _dev([30, 20, 0]), r.kt, r.vt), flux.FLUX_E_CAPACITY),
            (lambda: r.plan.flux_attn_decode_kvq(0, 3, r.f, r.rows(3, 4), r.kt, r.vt, _dev([30, 20, 1])), flux.FLUX_E_CAPACITY),
            (lambda: r.plan.flux_attn_decode_kvq(0, 2, -1, r.rows(2, 4), r.kt, r.vt, _dev([30, 20])), flux.FLUX_E_INVALID_ARG),
            (lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(2, 4), None, r.vt, _dev([30, 20])), flux.FLUX_E_INVALID_ARG)):
        with pytest.raises(flux.FluxError) as e:
            call()
        assert e.value.code == code
    for call in (lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(2, 8)[:, ::2], r.kt, r.vt, _dev([30, 20])),
                 lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(1, 4), r.kt, r.vt, _dev([30, 20])),
                 lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(2, 4).cpu(), r.kt, r.vt, _dev([30, 20])),
                 lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(2, 4), r.kt[:1], r.vt, _dev([30, 20])),
                 lambda: r.plan.flux_attn_decode_kvq(0, 2, r.f, r.rows(2, 4), r.kt, r.vt.cpu(), _dev([30, 20])),
                 lambda: r.plan.flux_kvq_store(0, r.f, k.float(), v, _dev([0, 1, 2]), _dev([30, 20]), r.kt, r.vt),
                 lambda: r.plan.flux_kvq_store(0, r.f, k, v[:-1], _dev([0, 1, 2]), _dev([30, 20]), r.kt, r.vt),
                 lambda: r.plan.flux_kvq_store(0, r.f, k, v, _dev([0, 1]), _dev([30, 20]), r.kt, r.vt)):
        with pytest.raises(ValueError):
            call()
    assert r.plan.flux_plan_status() == 0


# ---- decode -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 2), (7, 1), (28, 4), (8, 8), (16, 1), (9, 1), (32, 8), (36, 3)])
def test_decode_head_layouts(flux, fmt, Hq, Hkv):
    r = Rig(flux, fmt, Hq, Hkv, 20, 70, [1, 0, 1, 0, 1], 700)
    r.store([300, 611, 0, 37, 64])
    q, out = r.decode()
    r.check(q, out, "%s %d/%d" % (fmt, Hq, Hkv))
    rec = r.plan.flux_debug_dispatch(5)
    assert rec[:, 0].tolist() == [1, 0, 1, 0, 1] and rec[:, 3].tolist() == r.ctx
    assert rec[1].tolist()[4:] == [0, 20, 541, 611] and rec[3].tolist()[4:] == [0, 37, 0, 0]
    assert r.guards() and r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("S,W", [(0, 1), (2, 3), (64, 256), (5, 33), (128, 64)])
def test_decode_lengths_and_windows(flux, fmt, S, W, layout):
    lens = [1, 2, 15, 16, 17, 31, 33, 48, 63, 64, 65, 79, 80, 81, 127, 128, 129, 320, 321, 335, 336, 337, 400, 511, 512, 600]
    for mode in (0, 1):
        r = Rig(flux, fmt, 4, 2, S, W, [mode] * len(lens), 640, layout=layout, seed=S + W)
        r.store(lens)
        q, out = r.decode()
        r.check(q, out, "mode %d" % mode)
        assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_decode_steps_through_blocks_and_ring(flux, fmt):
    """Steps one token at a time across block and tile borders, by store and decode and by the step call: the same caches, and
    outputs within the tolerance (the step call cuts the work elsewhere)."""
    modes = [1, 0, 0, 1]
    r = Rig(flux, fmt, 8, 2, 16, 40, modes, 300, layout=1)
    s = Rig(flux, fmt, 8, 2, 16, 40, modes, 300, layout=1)
    k, v = r.rows(101 + 30 + 47), r.rows(101 + 30 + 47)
    r.store([101, 30, 47, 0], k, v)
    s.store([101, 30, 47, 0], k, v)
    for step in range(90):
        k, v = r.rows(4), r.rows(4)
        r.store([1] * 4, k, v)
        q, out = r.decode()
        s.hist = r.hist
        _, out2 = s.decode(q, step=(k, v))
        completes = any(n % 16 == 0 for n in r.ctx)
        for one, other in zip(r.load([0] * 4, r.ctx), s.load([0] * 4, r.ctx)):
            assert torch.equal(one, other), step
        if step % 9 == 0 or completes:
            r.check(q, out, "step %d" % step)
            s.check(q, out2, "step call %d" % step)
    assert r.guards() and s.guards() and r.plan.flux_plan_status() == 0 and s.plan.flux_plan_status() == 0


def test_step_skips_inactive_requests(flux):
    r = Rig(flux, "e4m3", 4, 2, 4, 8, [1, 1, 0], 100)
    r.store([20, 0, 33])
    before = [b[1].clone() for b in r.bufs]
    k, v = r.rows(3), r.rows(3)
    q = r.rows(3, 4)
    out = r.plan.flux_attn_decode_step_kvq(0, 3, r.f, q, k, v, r.kt, r.vt, _dev([21, 0, 34]))
    for h, x in zip(r.hist, (k, v)):
        h[0], h[2] = torch.cat([h[0], x[:1]]), torch.cat([h[2], x[2:]])
    r.check(q, out)
    assert torch.equal(before[0], r.bufs[0][1]) and torch.equal(before[1], r.bufs[1][1])
    # non-finite entries: flagged, stored as zeros
    k[0, 0, 3], v[2, 1, 7] = float("nan"), float("inf")
    out = r.plan.flux_attn_decode_step_kvq(0, 3, r.f, q, k, v, r.kt, r.vt, _dev([22, 0, 35]))
    assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_NONFINITE
    k[0, 0, 3] = v[2, 1, 7] = 0
    for h, x in zip(r.hist, (k, v)):
        h[0], h[2] = torch.cat([h[0], x[:1]]), torch.cat([h[2], x[2:]])
    r.check(q, out)
    # too long: flagged, nothing stored, a zero row
    out = r.plan.flux_attn_decode_step_kvq(0, 3, r.f, q, k, v, r.kt, r.vt, _dev([-5, 101, 36]))
    assert r.plan.flux_plan_status(raise_on_flag=False) == flux.FLUX_STATUS_BAD_LENGTH
    assert bool((out[:2] == 0).all()) and bool((out[2] != 0).any())
    assert torch.equal(before[0], r.bufs[0][1])


@pytest.mark.parametrize("fmt", FMTS)
def test_decode_long_context_and_large_batch(flux, fmt):
    r = Rig(flux, fmt, 8, 2, 128, 1024, [1, 0, 1], 20000, layout=1)
    r.store([20000, 19999, 1])
    q, out = r.decode()
    r.check(q, out, "long")
    assert r.plan.flux_plan_status() == 0
    B = 300
    lens = [(37 * i * i + i) % 200 for i in range(B)]
    r = Rig(flux, fmt, 4, 2, 16, 32, [i % 3 % 2 for i in range(B)], 200, layout=1)
    r.store(lens)
    q, out = r.decode()
    r.check(q, out, "wide")
    again = r.decode(q)[1]
    assert torch.equal(out, again) and r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (16, 1)])
def test_largest_batch_and_nobody_active(flux, Hq, Hkv):
    B = 1024
    r = Rig(flux, "int8", Hq, Hkv, 4, 8, [i % 2 for i in range(B)], 90, layout=1)
    q, out = r.decode()
    assert bool((out == 0).all())                       # no request has a token yet
    r.store([i % 5 * (i % 17) for i in range(B)])
    q, out = r.decode()
    r.check(q, out)
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_decode_magnitudes(flux, fmt):
    """Blocks of V whose scales differ by 2^80, sharp scores, tiny and zero queries."""
    r = Rig(flux, fmt, 4, 1, 4, 8, [1, 1, 1], 200)
    k, v = r.rows(450), r.rows(450)
    for j in range(0, 450, 16):
        v[j:j + 16] *= 2.0 ** ((j * 7) % 80 - 40)
        k[j:j + 16] *= 2.0 ** ((j * 5) % 7 - 3)
    v[160:176] = 0
    r.store([150, 150, 150], k, v)
    q = r.rows(3, 4)
    q[0, 0] = 0
    q[0, 1] *= 2.0 ** -90
    q[1] *= 8
    q[2, 0, 1:] *= 2.0 ** -20
    q[2, 3] *= 2.0 ** -8
    q, out = r.decode(q)
    r.check(q, out)
    assert r.plan.flux_plan_status() == 0


def test_decode_in_a_graph_on_another_stream(flux):
    """Capture a step (store and decode), replay it over a moving length, with a second plan's graph between the replays."""
    rigs = [Rig(flux, f, 8, 2, 16, 40, [1, 0], 300, layout=1, seed=9 + i) for i, f in enumerate(FMTS)]
    side = torch.cuda.Stream()
    work = []
    for r in rigs:
        r.store([70, 90])
        q, k, v, ctx, out = r.rows(2, 8), r.rows(2), r.rows(2), _dev([71, 91]), torch.zeros(2, 8, 128, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            r.plan.flux_attn_decode_step_kvq(0, 2, r.f, q, k, v, r.kt, r.vt, ctx, out)
        work.append((r, g, q, k, v, ctx, out))
    for step in range(30):
        for r, g, q, k, v, ctx, out in work:
            k.copy_(r.rows(2)); v.copy_(r.rows(2)); q.copy_(r.rows(2, 8))
            ctx.copy_(_dev([71 + step, 91 + step]))
            for h, x in zip(r.hist, (k, v)):
                h[0], h[1] = torch.cat([h[0], x[:1]]), torch.cat([h[1], x[1:]])
            g.replay()
        if step % 7 == 0 or step == 29:
            for r, g, q, k, v, ctx, out in work:
                r.check(q, out, "replay %d" % step)
    assert all(r.plan.flux_plan_status() == 0 for r in rigs)


def test_positions_loaded_are_recorded(flux):
    r = Rig(flux, "e4m3", 4, 2, 20, 70, [1, 0], 700)
    r.store([333, 611])
    bitmap = torch.zeros((2, 22), dtype=torch.int32, device=DEV)
    r.plan.flux_debug_touched(bitmap)
    r.decode()
    r.plan.flux_debug_touched(None)
    words = bitmap.cpu().numpy().view(np.uint32)
    seen = [[p for p in range(704) if words[b, p // 32] >> (p % 32) & 1] for b in range(2)]
    assert seen[0] == list(range(333))
    assert seen[1] == list(range(32)) + list(range(512, 611))      # strips of 32 that hold kept positions, and the tail


@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("fmt", FMTS)
def test_launch_overlap_gives_the_same_bits(flux, fmt, layers):
    """Steps of the layers one after another, call by call and as a replayed graph, with launch overlap on and off."""
    modes, lens = [1, 0, 0, 1, 1], [3000, 95, 700, 16, 0]
    rigs = [[Rig(flux, fmt, 8, 2, 16, 40, modes, 3200, layout=1, seed=layer) for layer in range(layers)] for _ in range(3)]
    first = [(r.rows(sum(lens)), r.rows(sum(lens))) for r in rigs[0]]
    for kind in range(3):
        for r, (k, v) in zip(rigs[kind], first):
            r.store(lens, k, v)
    for r in rigs[1] + rigs[2]:
        r.plan.flux_plan_set_launch_overlap(True)
    ctx = _dev([n + 1 if n else 0 for n in lens])
    q = [rigs[0][0].rows(5, 8) for _ in range(layers)]
    k, v = [rigs[0][0].rows(5) for _ in range(layers)], [rigs[0][0].rows(5) for _ in range(layers)]
    outs = [[torch.zeros(5, 8, 128, dtype=torch.bfloat16, device=DEV) for _ in range(layers)] for _ in range(3)]

    def step(kind):
        for layer, r in enumerate(rigs[kind]):
            r.plan.flux_attn_decode_step_kvq(0, 5, r.f, q[layer], k[layer], v[layer], r.kt, r.vt, ctx, outs[kind][layer])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(2)
    for n in range(40):
        for layer in range(layers):
            for t in (q[layer], k[layer], v[layer]):
                t.copy_(torch.randn(t.shape, generator=rigs[0][0].gen, device=DEV))
        ctx.copy_(_dev([m + 1 + n if m else 0 for m in lens]))
        step(0)
        step(1)
        graph.replay()
        for layer in range(layers):
            assert torch.equal(outs[0][layer], outs[1][layer]) and torch.equal(outs[0][layer], outs[2][layer]), (n, layer)
    assert all(r.plan.flux_plan_status() == 0 and r.guards() for kind in rigs for r in kind)
