"""The size of a page pool's scratch, which the library tells on the host (no device)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def flux():
    from paper_2604_07394_b200 import build, flux as f
    build.build()
    f.load()
    return f


def _scratch(flux, n_rows, cols, n_pages):
    s = flux.PagePoolStruct(None, None, None, None, n_rows, cols, n_pages, 16, 2)
    out = ctypes.c_size_t()
    flux._check(flux.load().flux_pages_scratch_size(ctypes.byref(s), ctypes.byref(out)))
    return out.value


def test_scratch_grows_with_the_rows_of_a_call_not_of_the_table(flux):
    """A call lists 4096 rows at most, so a table with one row per (layer, request) needs no more scratch than one of 4096 rows."""
    for cols in (40, 16384):
        most = _scratch(flux, 4096, cols, 100000)
        assert _scratch(flux, 4000, cols, 100000) < most == _scratch(flux, 4097, cols, 100000) == _scratch(flux, 65536, cols, 100000)
    # per listed row: three words, and a bit mask and a sum per 32 columns
    assert _scratch(flux, 4096, 16384, 1024) < 4096 * (3 * 4 + 512 * 8) + 1024
