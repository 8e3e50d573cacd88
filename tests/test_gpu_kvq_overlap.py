"""Launch overlap of the 8-bit decode beside launches that write what it reads."""
import pytest
import torch

from tests.test_gpu_kvq import DEV, FMTS, Rig, _dev, flux  # noqa: F401 (flux: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (16, 1)])
@pytest.mark.parametrize("fmt", FMTS)
def test_query_rows_come_from_the_launch_before(flux, fmt, Hq, Hkv):
    """A chain of decodes whose query rows are the output rows of the launch before: the same bits with overlap on and off, call by call
    and replayed."""
    modes, lens = [1, 0, 1], [2500, 700, 33]
    r = Rig(flux, fmt, Hq, Hkv, 16, 40, modes, 3000, layout=1)
    r.store(lens)
    ctx = _dev(lens)
    bufs = [torch.zeros(3, Hq, 128, dtype=torch.bfloat16, device=DEV) for _ in range(31)]

    def chain():
        for a, b in zip(bufs, bufs[1:]):
            r.plan.flux_attn_decode_kvq(0, 3, r.f, a, r.kt, r.vt, ctx, b)

    def run(replay=None):
        for b in bufs[1:]:
            b.fill_(float("nan"))
        torch.cuda.synchronize()
        (replay or chain)()
        torch.cuda.synchronize()
        return [b.clone() for b in bufs[1:]]

    bufs[0].copy_(r.rows(3, Hq) * 4)
    want = run()
    assert all(bool(torch.isfinite(x).all()) for x in want)
    r.plan.flux_plan_set_launch_overlap(True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(want, run()))
        assert all(torch.equal(x, y) for x, y in zip(want, run(graph.replay)))
    assert r.plan.flux_plan_status() == 0
