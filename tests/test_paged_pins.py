"""Pins of the paged-cache oracle, and of what the library decides on the host (no device)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged


@pytest.fixture(scope="module")
def flux():
    from paper_2604_07394_b200 import build, flux as f
    build.build()
    f.load()
    return f


def test_norm_and_rotation_closed_forms():
    x = np.zeros((2, 1, 8))
    x[:, 0, 0], x[:, 0, 4], x[:, 0, 6] = 3.0, 4.0, 1.0
    # a quarter of a turn per position: (3, 4) -> (-4, 3); two positions: (-3, -4); channel 6 is its own pair's second half
    y, mag = paged.turned(x, [1, 2], [np.pi / 2, 0, 0, 0])
    assert np.allclose(y[0, 0, [0, 4, 6]], [-4, 3, 1]) and np.allclose(y[1, 0, [0, 4, 6]], [-3, -4, 1])
    assert np.allclose(mag[0, 0, [0, 4, 6]], [7, 7, 1])
    z, _ = paged.turned(x, [1, 2], [np.pi / 2, 0, 0, 0], pairs=True)          # neighbours: (3, 0) -> (0, 3)
    assert np.allclose(z[0, 0, [0, 1, 4]], [0, 3, 4])
    # the norm: rows of root mean square 1, weights as they are, an offset added
    w = np.arange(8.0)
    n, _ = paged.turned(x, [0, 0], [], weight=w, eps=0.0, offset=1.0)
    assert np.allclose(n[0, 0], x[0, 0] / np.sqrt(26 / 8) * (w + 1))
    # rotations keep lengths, and scores depend on the distance of positions alone
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
    f = [1.0, 0.3, 0.01, 0.002]
    s = [(paged.turned(q, [a], f)[0] * paged.turned(k, [b], f)[0]).sum() for a, b in ((5, 3), (105, 103), (2, 0))]
    assert np.allclose(s, s[0]) and np.allclose(np.linalg.norm(paged.turned(q, [77], f)[0]), np.linalg.norm(q))


def _pool(rows, pages=10, page=4):
    table = np.full((len(rows), 4), -1)
    for r, entries in enumerate(rows):
        table[r, :len(entries)] = entries
    refs = np.bincount(table[table >= 0], minlength=pages)
    data = np.arange(pages * page, dtype=np.float64).reshape(1, pages, page)
    return paged.Pool(table, refs, data, page)


def test_reserve_by_hand():
    p = _pool([[7, 2], [7, 5], [0]])
    # row 0 (6 tokens, page 2 its own) to 9: one page more; row 1 at a page's end: one page; row 2 begins its only page anew
    assert p.reserve([0, 1, 2], [6, 8, 0], [9, 9, 1]) == [1, 1, 1]
    assert p.table.tolist() == [[7, 2, 1, -1], [7, 5, 3, -1], [0, -1, -1, -1]] and p.refs.tolist() == [1, 1, 1, 1, 0, 1, 0, 2, 0, 0]
    # both rows share page 7 and begin to write inside it: row 0 gets a copy of its three tokens, row 1 keeps it
    p = _pool([[7], [7]])
    assert p.reserve([0, 1], [3, 2], [4, 3]) == [1, 1]
    assert p.table[:, 0].tolist() == [0, 7] and p.refs[[0, 7]].tolist() == [1, 1] and p.data[0, 0].tolist() == [28, 29, 30, 3]
    # a third holder who is not listed: both are copied
    p = _pool([[7], [7], [7]])
    assert p.reserve([0, 1], [3, 2], [4, 3]) == [1, 1] and p.table[:, 0].tolist() == [0, 1, 7] and p.refs[7] == 1
    # pages run out: who comes behind gets nothing either
    p = _pool([[0, 1, 2], [3, 4], []], pages=7)
    assert p.reserve([0, 1, 2], [12, 8, 0], [13, 16, 1]) == [1, 0, 0] and p.no_pages and p.table[1].tolist() == [3, 4, -1, -1]


def test_fork_release_compact_by_hand():
    p = _pool([[1, 2, 3], [4], [5, 6]])
    p.fork([0, 1], [1, 0], [5, 4])                  # rows change places, row 0's second page with it, its third is gone
    assert p.table.tolist() == [[4, -1, -1, -1], [1, 2, -1, -1], [5, 6, -1, -1]] and p.refs.tolist() == [0, 1, 1, 0, 1, 1, 1, 0, 0, 0]
    p.release([2, 1], [1, 0], [8, 4])               # page 5 holds position 0 too; page 1 lies inside
    assert p.table.tolist() == [[4, -1, -1, -1], [-1, 2, -1, -1], [5, -1, -1, -1]] and p.refs.sum() == 3
    to, n = p.compact()
    assert n == 3 and to.tolist() == [-1, -1, 2, -1, 0, 1, -1, -1, -1, -1]
    assert p.table.tolist() == [[0, -1, -1, -1], [-1, 2, -1, -1], [1, -1, -1, -1]] and p.data[0, :3, 0].tolist() == [16, 20, 8]


def test_fractions_of_a_turn(flux):
    f = np.array([1.0, 0.25, 1e-6, 0.0, 2 * np.pi, np.pi / 2, -np.pi / 2, 700.0])
    got = flux.flux_rope_freqs(f)
    turns = f / (2 * np.pi)
    want = turns - np.floor(turns)
    err = np.abs(got.astype(np.float64) / 2.0 ** 64 - want)
    assert (np.minimum(err, 1 - err) < 1e-14 * np.maximum(1, np.abs(turns))).all()
    assert got[3] == 0 and flux.flux_rope_freqs(np.array([])).size == 0
    for bad in ([np.nan], [np.inf], np.ones(65)):
        with pytest.raises(flux.FluxError) as e:
            flux.flux_rope_freqs(np.array(bad))
        assert e.value.code == flux.FLUX_E_INVALID_ARG


def test_scratch_size_and_pool_limits(flux):
    def size(**kw):
        s = flux.PagePoolStruct(None, None, None, None, 4, 100, 1000, 16, 2)
        for k, v in kw.items():
            setattr(s, k, v)
        out = ctypes.c_size_t()
        flux._check(flux.load().flux_pages_scratch_size(ctypes.byref(s), ctypes.byref(out)))
        return out.value

    assert 0 < size() < 1 << 14 < size(n_pages=1 << 20) < 1 << 20
    for kw, code in ((dict(page_size=24), flux.FLUX_E_UNSUPPORTED_SHAPE), (dict(page_size=8), flux.FLUX_E_UNSUPPORTED_SHAPE),
                     (dict(page_size=512), flux.FLUX_E_UNSUPPORTED_SHAPE), (dict(n_pages=0), flux.FLUX_E_CAPACITY),
                     (dict(n_pages=(1 << 24) + 1), flux.FLUX_E_CAPACITY), (dict(max_pages=0), flux.FLUX_E_CAPACITY),
                     (dict(max_pages=(1 << 26) + 1), flux.FLUX_E_CAPACITY), (dict(n_rows=0), flux.FLUX_E_INVALID_ARG),
                     (dict(n_slabs=-1), flux.FLUX_E_INVALID_ARG)):
        with pytest.raises(flux.FluxError) as e:
            size(**kw)
        assert e.value.code == code, kw


def test_calls_without_a_plan_are_refused(flux):
    L, none = flux.load(), None
    bad = flux.FLUX_E_INVALID_ARG
    assert L.flux_qk_norm_rope(none, none, none, none, 0, 0, 1, none, none, none, 0, 0, none) == bad
    assert L.flux_paged_store(none, 1, none, none, none, none, 0, 0, 0, 1, none, none, none, none, none, none) == bad
    assert L.flux_paged_load(none, 1, none, none, 1, none, none, none, none, none) == bad
    assert L.flux_attn_decode_paged(none, 0, 1, none, 0, none, none, none, none) == bad
    assert L.flux_attn_decode_step_paged(none, 0, 1, none, none, none, none, 0, 0, 0, none, none, none, none) == bad
    assert L.flux_pages_reserve(none, none, 1, none, none, none, none, none) == bad
    assert L.flux_pages_fork(none, none, 1, none, none, none, none) == bad
    assert L.flux_pages_release(none, none, 1, none, none, none, none) == bad
    assert L.flux_pages_compact(none, none, none, none, none) == bad


def test_tensors_of_another_form_are_refused(flux):
    pool = torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    table = torch.zeros(3, 2, dtype=torch.int32)
    for k, v, t in ((pool.float(), pool, table), (pool, pool[:3], table), (pool[:, ::2], pool[:, ::2], table), (pool[0], pool[0], table),
                    (pool[..., :64].contiguous(), pool[..., :64].contiguous(), table), (pool, pool, table[0]), (pool, pool, table.long())):
        with pytest.raises(ValueError):
            flux.Pages(k, v, t)
    refs = torch.zeros(4, dtype=torch.int32)
    for t, r, slabs in ((table, refs[:3], [pool]), (table[0], refs, [pool]), (table, refs, []), (table, refs, [pool, pool[:3]]), (table, refs, [pool.float()])):
        with pytest.raises(ValueError):
            flux.PagePool(t, r, slabs)
    with pytest.raises(ValueError):
        flux.Rope(np.ones((2, 2)), device="cpu")
    with pytest.raises(ValueError):
        flux.Rope(np.ones(64), q_weight=torch.ones(64, dtype=torch.bfloat16), device="cpu")
    with pytest.raises(ValueError):
        flux.Rope(np.ones(64), k_weight=torch.ones(128), device="cpu")
