"""CPU pins of the 8-bit cache oracle (oracle/kvq.py), and the refusals of the calls that need no device."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kvq
from paper_2604_07394_b200 import build as flux_build
from paper_2604_07394_b200 import flux


def test_round_e4m3_against_the_cast_and_by_hand():
    # every number of the type is a fixed point; the middles go to the even neighbour
    all_codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    all_codes = np.unique(all_codes[np.isfinite(all_codes)])
    assert np.array_equal(kvq.round_e4m3(all_codes), all_codes) and all_codes.max() == 448
    x = np.random.default_rng(5).standard_normal(200000) * np.exp(np.random.default_rng(6).uniform(-8, 4, 200000))
    x = np.clip(x, -448, 448).astype(np.float32)
    mid = ((all_codes[1:] + all_codes[:-1]) / 2).astype(np.float32)
    for y in (x, mid):
        assert np.array_equal(kvq.round_e4m3(y.astype(np.float64)), torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy())
    assert kvq.round_e4m3(np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10])).tolist() == [16.0, 20.0, 0.0, 2.0 ** -8]


def test_scales_by_hand():
    assert kvq.scale(448.0, "e4m3") == 1.0 and kvq.scale(449.0, "e4m3") == 2.0 and kvq.scale(224.0, "e4m3") == 0.5
    assert kvq.scale(1.75, "e4m3") == 2.0 ** -8 and kvq.scale(1.7578125, "e4m3") == 2.0 ** -7
    assert kvq.scale(0.0, "e4m3") == kvq.scale(0.0, "int8") == 1.0
    assert kvq.scale(127.0, "int8") == 1.0 and kvq.scale(1.0, "int8") == float(np.float32(1 / 127))
    assert kvq.scale(1e-38, "e4m3") == kvq.scale(1e-38, "int8") == 2.0 ** -100
    top = 3.3895313892515355e38                                        # 0x7f7f: the largest bf16, 1.99 * 2^127
    assert kvq.scale(top, "e4m3") == 2.0 ** 119 and kvq.block_values(np.array([top, -top, 1e38]), "e4m3").tolist()[:2] == [448 * 2.0 ** 119, -448 * 2.0 ** 119]


def test_cache_values_blocks_tail_and_error_bounds():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 2, 128))
    for fmt in ("e4m3", "int8"):
        y = kvq.cache_values(x, fmt)
        assert np.array_equal(y[32:], x[32:])                       # the incomplete block is as it was
        for j in (0, 1):
            for h in (0, 1):
                b, c = x[16 * j:16 * j + 16, h], y[16 * j:16 * j + 16, h]
                top = np.abs(b).max()
                # half a step: int8 amax / 254; e4m3 2^-4 relative, or half a subnormal step of the scale
                bound = top / 254 * (1 + 1e-6) if fmt == "int8" else np.maximum(np.abs(b) * 2.0 ** -4, kvq.scale(top, fmt) * 2.0 ** -10)
                assert (np.abs(b - c) <= bound).all() and np.abs(b - c).max() > 0
    x[3, 1, 7], x[20, 0, 0] = np.nan, -np.inf
    z = x.copy()
    z[3, 1, 7] = z[20, 0, 0] = 0
    assert np.array_equal(kvq.cache_values(x, "int8"), kvq.cache_values(z, "int8"))


def test_attend_closed_forms():
    q = np.zeros((2, 4))
    k = np.zeros((3, 1, 4))
    v = np.arange(12.0).reshape(3, 1, 4) - 5
    out, mag_v, mag, p = kvq.attend(q, k, v, 1.0)
    assert np.allclose(out, v.mean(0)) and np.allclose(mag_v, np.abs(v).mean(0)) and (mag == 0).all() and np.allclose(p, 1 / 3)
    q[0, 0], k[1, 0, 0] = 1.0, np.log(2.0)
    assert np.allclose(kvq.attend(q, k, v, 1.0)[3][0], [0.25, 0.5, 0.25])
    assert kvq.kept(10, False, 2, 3).tolist() == [0, 1, 7, 8, 9] and len(kvq.kept(10, True, 2, 3)) == 10


@pytest.fixture(scope="module")
def lib():
    flux_build.build()
    return flux.load()


def test_cache_size(lib):
    cfg = flux.make_config(2, 8, 2, 64, 256, 1, 4096)
    tile = (2 * 2 * (32 * 128 + 16) + 127) // 128 * 128      # two strips of two heads, codes and scales, padded to 128 bytes
    tail = 2 * 16 * 256
    assert flux.flux_kvq_cache_size(cfg, False, 0) == tail
    assert flux.flux_kvq_cache_size(cfg, False, 1) == tail + tile
    assert flux.flux_kvq_cache_size(cfg, False, 4096) == tail + 64 * tile
    # sink 64 = 1 tile; a window of 256 positions can touch 5 tiles
    assert flux.flux_kvq_cache_size(cfg, True, 4096) == tail + 6 * tile
    assert flux.flux_kvq_cache_size(cfg, True, 100) == tail + 2 * tile
    for bad in (-1, 4097):
        with pytest.raises(flux.FluxError) as e:
            flux.flux_kvq_cache_size(cfg, False, bad)
        assert e.value.code == flux.FLUX_E_CAPACITY
    assert lib.flux_kvq_cache_size(ctypes.byref(cfg), 0, 1, None) == flux.FLUX_E_INVALID_ARG
    assert lib.flux_kvq_cache_size(None, 0, 1, ctypes.byref(ctypes.c_size_t())) == flux.FLUX_E_INVALID_ARG


def test_calls_without_a_plan_are_refused(lib):
    assert lib.flux_kvq_store(None, 0, 1, 0, None, None, 0, 0, 1, None, None, None, None, None) == flux.FLUX_E_INVALID_ARG
    assert lib.flux_kvq_load(None, 0, 1, 0, None, None, None, 1, None, None, None, None, None) == flux.FLUX_E_INVALID_ARG
    assert lib.flux_attn_decode_kvq(None, 0, 1, 0, None, None, None, None, None, None) == flux.FLUX_E_INVALID_ARG
    assert lib.flux_attn_decode_step_kvq(None, 0, 1, 0, None, None, None, None, None, None, None, None) == flux.FLUX_E_INVALID_ARG


def test_binding_refuses_other_types_and_layouts():
    ok = torch.zeros(5, 2, 128, dtype=torch.bfloat16)
    assert flux._rows(ok, 2, "k") == 256
    assert flux._rows(torch.zeros(5, 6, 128, dtype=torch.bfloat16)[:, 2:4], 2, "k") == 768      # a slice of a fused projection
    for bad in (ok.float(), ok[:, :1], ok[:, :, :64], ok.transpose(0, 1), ok[0], ok.permute(0, 2, 1).contiguous().permute(0, 2, 1)):
        with pytest.raises(ValueError):
            flux._rows(bad, 2, "k")
    with pytest.raises(ValueError):
        flux._int32(torch.zeros(4), 4, "pos")
    with pytest.raises(ValueError):
        flux._int32(torch.zeros(4, dtype=torch.int32), 5, "pos")
    with pytest.raises(ValueError):
        flux._int32(torch.zeros(8, dtype=torch.int32)[::2], 4, "pos")


def test_binding_refuses_host_tensors_and_short_tables():
    """A host address must never reach a kernel, nor a table with fewer entries than requests."""
    import pytest
    torch = pytest.importorskip("torch")
    from paper_2604_07394_b200 import flux
    rows = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    for call in (lambda: flux._rows(rows, 2, "k", 0), lambda: flux._flat_rows(rows, 4, 2, "q", 0),
                 lambda: flux._int32(torch.zeros(3, dtype=torch.int32), 3, "pos", 0),
                 lambda: flux._table(torch.zeros(3, dtype=torch.int64), 3, "k_caches", 0)):
        with pytest.raises(ValueError, match="cuda:0"):
            call()
    # on the device they ask for (a host tensor's is -1) the same arguments pass, but for sizes and types
    assert flux._rows(rows, 2, "k", -1) == 256 and flux._flat_rows(rows, 4, 2, "q", -1) == rows.data_ptr()
    table = torch.zeros(3, dtype=torch.int64)
    assert flux._table(table, 3, "k_caches", -1) == table.data_ptr() and flux._table(None, 3, "k_caches", -1) is None
    for t, n in ((table, 4), (table.int(), 3), (table.repeat(2)[::2], 3)):
        with pytest.raises(ValueError):
            flux._table(t, n, "k_caches", -1)
