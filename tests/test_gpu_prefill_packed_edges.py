"""Packed prefill: dispatch records of requests that no launch has work for, and how far a non-finite V entry reaches."""
import numpy as np
import pytest
import torch

from tests.test_gpu_prefill_packed import DEV, _cum, _plan, _rows, flux  # noqa: F401 (flux: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,busy", [(130, [0, 129]), (64, []), (200, [70]), (65, [64]), (3, []), (192, list(range(64, 128)))])
def test_records_of_requests_without_new_tokens(flux, B, busy):
    """Every request of the call has a record of this call (mode -1: skipped), also where a launch's whole share has nothing to do."""
    plan = _plan(flux, 4, 2, 8, 16, [i % 2 for i in range(B)], 40)
    full = [3] * B
    q, k = _rows(3 * B, 4, 1), _rows(3 * B, 2, 2)
    plan.flux_attn_prefill_packed(0, q, k, k, _cum(full))                  # fills the records
    assert plan.flux_debug_dispatch(B)[:, 0].tolist() == [i % 2 for i in range(B)]
    new = [5 if b in busy else 0 for b in range(B)]
    want = plan.flux_attn_prefill_packed(0, q, k, k, _cum(new))
    rec = plan.flux_debug_dispatch(B)
    assert len(rec) == B
    assert rec[:, 0].tolist() == [b % 2 if b in busy else -1 for b in range(B)]
    assert rec[:, 2].tolist() == list(range(B)) and rec[:, 3].tolist() == new
    assert torch.equal(want[:sum(new)], plan.flux_attn_prefill_packed(0, q, k, k, _cum(new))[:sum(new)])
    assert plan.flux_plan_status() == 0


def test_records_after_a_larger_call(flux):
    """An empty call replaces the records of the call before it, count and all."""
    plan = _plan(flux, 4, 2, 8, 16, [1] * 5, 40)
    q, k = _rows(20, 4, 1), _rows(20, 2, 2)
    plan.flux_attn_prefill_packed(0, q, k, k, [0, 4, 8, 12, 16, 20])
    plan.flux_attn_prefill_packed(0, q, k, k, [7, 7, 7])
    rec = plan.flux_debug_dispatch(5)
    assert rec.shape[0] == 2 and rec[:, 0].tolist() == [-1, -1] and rec[:, 2].tolist() == [0, 1]
    assert plan.flux_plan_status() == 0


def _tiles(rows, past, keys, fa, S, W):
    """128-position key tiles that the query tiles holding the given new rows walk."""
    first, last = past + min(rows) // 128 * 128, min(past + max(rows) // 128 * 128 + 127, keys - 1)
    end = last // 128 + 1
    if fa:
        return set(range(end))
    return set(range(min(-(-S // 128), end))) | set(range(max(0, first - W + 1) // 128, end))


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (7, 1), (3, 3)])
@pytest.mark.parametrize("new,past", [(400, 0), (300, 50), (129, 1000), (3, 4000)])
def test_how_far_a_non_finite_value_reaches(flux, Hq, Hkv, new, past):
    """An infinite or NaN V entry: rows that keep it are non-finite in its channel; it reaches no row but those whose query tile (in the
    last head of an odd group: its partner too) walks the entry's key tile; everything else keeps its bits."""
    S, W, keys = 130, 200, new + past
    G = Hq // Hkv
    q, k, v = _rows(new, Hq, 1), _rows(keys, Hkv, 2), _rows(keys, Hkv, 3)
    n_qt = -(-new // 128)
    for fa in (True, False):
        plan = _plan(flux, Hq, Hkv, S, W, [int(fa)], keys)
        want = plan.flux_attn_prefill_packed(0, q, k, v, [0, new], [0, keys])
        for at, val in ((keys - 1, float("inf")), (past + new // 2, float("nan")), (150, -float("inf")), (past, float("inf"))):
            bad = v.clone()
            bad[at, Hkv - 1, 77] = val
            out = plan.flux_attn_prefill_packed(0, q, k, bad, [0, new], [0, keys])
            for h in range(Hq):
                same = (out[:, h] == want[:, h]).all(1).cpu().numpy()
                finite = torch.isfinite(out[:, h, 77]).cpu().numpy()
                others = torch.cat([out[:, h, :77], out[:, h, 78:]], 1) == torch.cat([want[:, h, :77], want[:, h, 78:]], 1)
                assert bool(others.all())
                if h // G != Hkv - 1:
                    assert same.all()
                    continue
                for t in range(n_qt):
                    rows = [t * 128, min(t * 128 + 127, new - 1)]
                    if G % 2 and h % G == G - 1:                   # left-over head: tiles in pairs, counted from the last one
                        pair = (n_qt - 1 - t) // 2
                        low = max(n_qt - 2 - 2 * pair, 0)
                        rows = [low * 128, min((n_qt - 1 - 2 * pair) * 128 + 127, new - 1)]
                    if at // 128 not in _tiles(rows, past, keys, fa, S, W):
                        assert same[t * 128:t * 128 + 128].all(), (fa, at, h, t)
                for r in range(new):
                    if at <= past + r and (fa or at < S or at > past + r - W):
                        assert not finite[r], (fa, at, h, r)
        assert plan.flux_plan_status() == 0


def test_single_kv_head_with_an_odd_head_stride(flux):
    plan = _plan(flux, 4, 1, 8, 16, [1, 0], 100)
    q, k, v = _rows(150, 4, 1), _rows(150, 1, 2), _rows(150, 1, 3)
    want = plan.flux_attn_prefill_packed(0, q, k, v, [0, 90, 150])
    shown = [x.view(1, 150, 128).transpose(0, 1) for x in (k, v)]
    assert shown[0].stride() == (128, 150 * 128, 1)
    assert torch.equal(plan.flux_attn_prefill_packed(0, q, *shown, [0, 90, 150]), want)
    assert plan.flux_plan_status() == 0
