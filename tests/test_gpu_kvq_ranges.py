"""8-bit decode over the whole range of V: scales from 2^-100 to 2^119, blocks of zeros, and queries of every magnitude.  Attention is
linear in V, so the bounds of tests/test_gpu_kvq.py (Rig.check; a block of zeros enters them with the smallest scale) hold at every size."""
import numpy as np
import pytest
import torch

from oracle import kvq
from tests.test_gpu_kvq import DEV, FMTS, Rig, flux  # noqa: F401 (flux: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FMTS)
def test_many_keys_at_the_smallest_scale(flux, fmt):
    """2^18 and more keys of equal score whose scale is 2^-100: the row sum of their weights has to stay finite."""
    n = (1 << 18) + (1 << 15)
    r = Rig(flux, fmt, 1, 1, 4, 8, [1], n)
    k = torch.zeros(n, 1, 128, dtype=torch.bfloat16, device=DEV)
    v = (torch.randn(n, 1, 128, generator=r.gen, device=DEV) + 2).mul_(2.0 ** -96).to(torch.bfloat16)
    r.store([n], k, v)
    q, out = r.decode()
    assert torch.isfinite(out).all()
    held = kvq.cache_values(v.double().cpu().numpy(), fmt)
    # equal weights, exact in fp16: half a step of the output, and at most 16 x 17 additions in a warp (some 250 keys, 16 to a product)
    # and 160 of parts, each off by 2^-23 where it is cut off instead of rounded
    ref = held.mean(0)
    err = np.abs(out[0].double().cpu().numpy() - ref)
    assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -14 * np.abs(held).mean(0)).all()
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (16, 1)])
@pytest.mark.parametrize("fmt", FMTS)
def test_scales_further_apart_than_fp32_reaches(flux, fmt, Hq, Hkv):
    """Blocks of V of size 2^110 beside blocks of 2^-95, scores alike: the small ones' keys count in the row sum all the same."""
    lens = [64, 500, 33, 1700]
    r = Rig(flux, fmt, Hq, Hkv, 4, 8, [1] * 4, 2000)
    k, v = r.rows(sum(lens)), r.rows(sum(lens))
    first = np.cumsum([0] + lens)
    for b, n in enumerate(lens):
        for j in range(0, n, 16):
            v[first[b] + j:min(first[b] + j + 16, first[b] + n)] *= 2.0 ** (110 if (j // 16) % 3 == b % 3 else -95)
    r.store(lens, k, v)
    q, out = r.decode()
    r.check(q, out)
    assert r.plan.flux_plan_status() == 0


def _zeros_among_small_values(flux, fmt, Hq, Hkv, size, sink, step=False):
    lens = [48, 333, 64, 700, 2900, 100] + [160] * 20
    B = len(lens)
    r = Rig(flux, fmt, Hq, Hkv, 4, 8, [1] * B, 3000, seed=int(Hq))
    k, v, q = r.rows(sum(lens)), r.rows(sum(lens)), r.rows(B, Hq)
    v *= size
    first = np.cumsum([0] + lens)
    if sink:                                   # keys of the zero blocks score about 11 (nats) above the others
        q[:, :, 0] = 8.0
        k[:, :, 0] = 0.0
    for b in range(B):
        for j in ([0], [0, 160], [16], [32, 48, 64], [0, 1600], range(0, 96, 16))[b % 6]:
            if j + 16 <= lens[b]:
                v[first[b] + j:first[b] + j + 16] = 0
                if sink:
                    k[first[b] + j:first[b] + j + 16, :, 0] = 16.0
    r.store(lens, k, v)
    if not step:
        return r, *r.decode(q)
    kn, vn = r.rows(B), r.rows(B) * size
    for h, x in zip(r.hist, (kn, vn)):
        for b in range(B):
            h[b] = torch.cat([h[b], x[b:b + 1]])
    return r, *r.decode(q, (kn, vn))


@pytest.mark.parametrize("sink", [False, True])
@pytest.mark.parametrize("size", [1.0, 1e-3, 2.0 ** -24, 2.0 ** -30, 2.0 ** -60])
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (16, 1)])
@pytest.mark.parametrize("fmt", FMTS)
def test_blocks_of_zeros_leave_small_values_their_precision(flux, fmt, Hq, Hkv, size, sink):
    """Blocks of zeros (padding, cleared entries) ahead of, between and behind blocks of V of any size."""
    r, q, out = _zeros_among_small_values(flux, fmt, Hq, Hkv, size, sink)
    r.check(q, out, "size %g" % size)
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_blocks_of_zeros_in_the_step_call(flux, fmt):
    r, q, out = _zeros_among_small_values(flux, fmt, 8, 2, 2.0 ** -30, True, step=True)
    r.check(q, out)
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_all_zero_requests_and_a_block_that_becomes_zero(flux, fmt):
    """V of zeros throughout gives zero rows, whatever the scores; loaded values are zeros; steps that complete a block of zeros."""
    r = Rig(flux, fmt, 8, 2, 4, 8, [1, 0, 1], 700)
    lens = [600, 300, 15]
    k, v = r.rows(915) * 4, torch.zeros(915, 2, 128, dtype=torch.bfloat16, device=DEV)
    v[::2] = -v[::2]                          # -0.0 too
    r.store(lens, k, v)
    ko, vo = r.load([0, 0, 0], lens)
    assert bool((vo == 0).all())
    q, out = r.decode()
    assert bool((out == 0).all())
    for _ in range(18):                        # the third request's first block is completed by the first step, with zeros
        kn, vn = r.rows(3), torch.zeros(3, 2, 128, dtype=torch.bfloat16, device=DEV)
        for h, x in zip(r.hist, (kn, vn)):
            for b in range(3):
                h[b] = torch.cat([h[b], x[b:b + 1]])
        q, out = r.decode(step=(kn, vn))
        assert bool((out == 0).all())
    v2 = r.rows(3 * 40) * 2.0 ** -40           # small values behind all those zeros
    r.store([40] * 3, r.rows(120), v2)
    q, out = r.decode()
    r.check(q, out)
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_queries_of_every_magnitude(flux, fmt):
    """Query rows up to the largest bf16 over keys so small, or zero, that the scores stay finite."""
    r = Rig(flux, fmt, 8, 2, 4, 8, [1, 1], 300)
    k, v = r.rows(400) * 2.0 ** -90, r.rows(400)
    k[200:] = 0
    r.store([200, 200], k, v)
    q = r.rows(2, 8)
    for h, e in enumerate((90, 95, 88, 92, 60, 0, -60, -120)):
        q[0, h] *= 2.0 ** e
    for h, e in enumerate((127, 126, 120, 117, 116, 100, 60, -126)):
        q[1, h] = (q[1, h].sign() * 2.0 ** e).to(torch.bfloat16)
    q[1, 0, ::3] = torch.finfo(torch.bfloat16).max
    q, out = r.decode(q)
    r.check(q, out)
    assert r.plan.flux_plan_status() == 0


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (16, 1)])
@pytest.mark.parametrize("fmt", FMTS)
def test_a_key_that_outweighs_the_rest_comes_out_as_it_is(flux, fmt, Hq, Hkv):
    """Its weight is the row sum but for 2^-40 (here the newest of 1 to 15 keys, in bf16), so the output is its V row: weight, row sum and
    quotient are off by 2^-20 at most, which does not move a bf16 number to another."""
    lens = [1 + i % 15 for i in range(60)]
    r = Rig(flux, fmt, Hq, Hkv, 4, 8, [1] * 60, 100)
    k, v = r.rows(sum(lens)) * 0.125, r.rows(sum(lens))
    q = r.rows(60, Hq)
    q[:, :, 0] = 23.0
    newest = np.cumsum(lens) - 1
    k[:, :, 0] = 0.0
    k[newest, :, 0] = 37.0
    r.store(lens, k, v)
    s = torch.einsum("bhd,bhd->bh", q.double(), k[newest].double().repeat_interleave(Hq // Hkv, 1)) / np.sqrt(128)
    assert float(s.min()) > 60                 # the other keys' scores stay below 20: N(0, 1) entries 0.125 apart, a few channels 36 times that
    q, out = r.decode(q)
    assert torch.equal(out, v[newest].repeat_interleave(Hq // Hkv, 1))
    assert r.plan.flux_plan_status() == 0
