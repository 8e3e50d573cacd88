"""8-bit decode over the whole range of V: scales from 2^-100 to 2^119.  Attention is linear in V, so the bounds of tests/test_gpu_kvq.py
(Rig.check) hold at every size."""
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
