"""Packed prefill: dispatch records of requests that no launch has work for."""
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
