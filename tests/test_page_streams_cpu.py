"""Which paged decodes wait for the launch before them although launch overlap is on: those right behind a page call in their stream."""
import ctypes
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_07394_b200", "csrc")


@pytest.fixture()
def streams(tmp_path):
    src = tmp_path / "shim.cpp"
    src.write_text('#include "flux_stream_set.h"\nstatic flux::StreamSet s;\nextern "C" { void clear() { s.n = 0; } void add(void *p) { s.add(p); }\n'
                   'int take(void *p) { return s.take(p); } int most() { return flux::StreamSet::kMost; } }\n')
    lib = tmp_path / "shim.so"
    subprocess.check_call(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(lib), str(src)])
    L = ctypes.CDLL(str(lib))
    for name in ("add", "take"):
        getattr(L, name).argtypes = [ctypes.c_void_p]
    L.clear()
    return L


def test_one_decode_per_stream(streams):
    assert not streams.take(None) and not streams.take(0x100)
    streams.add(0x100)
    streams.add(0x100)
    streams.add(0x200)
    assert not streams.take(0x300)
    assert streams.take(0x100) and not streams.take(0x100)          # once, however many page calls there were
    assert streams.take(0x200) and not streams.take(0x200)
    streams.add(1)                                                  # the default stream has two names
    assert streams.take(None) and not streams.take(1)


def test_more_streams_than_are_kept(streams):
    most = streams.most()
    for i in range(most):
        streams.add(0x1000 + i)
    assert not streams.take(0x10) and streams.take(0x1000 + most // 2) and not streams.take(0x1000 + most // 2)
    streams.add(0x1000 + most // 2)
    streams.add(0x2000)                                             # one too many: every decode waits
    assert streams.take(0x2000) and streams.take(0x10) and streams.take(0x10)
    streams.add(0x3000)
    assert streams.take(0x1000)


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))


def test_page_calls_are_noted_and_the_decode_asks():
    pages, decode = _code("flux_pages.cu"), _code("flux_decode_paged.cu")
    # all launches of the page calls go through one function, which notes the stream
    assert pages.count("cudaLaunchKernelEx") == 1 and "<<<" not in pages
    assert re.search(r"page_calls\.add\(st\);\s*return check_cuda\(cudaLaunchKernelEx", pages)
    assert re.search(r"const bool (\w+) = p->page_calls\.take\(st\);\s*a\.overlap = p->launch_overlap && !\1;", decode)
    # what is read ahead of the wait with overlap is behind it without
    assert re.search(r"if \(!a\.overlap\) \{\s*wait\(\);\s*release\(\);\s*\}", decode)
