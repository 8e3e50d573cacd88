"""Rules of programmatic launches, held by the sources: what a kernel may do while the launches before it are still running."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2604_07394_b200", "csrc")


def _code(name):
    text = open(os.path.join(CSRC, name)).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return re.sub(r"//[^\n]*", "", text)


def test_rows_of_the_launch_before_are_not_read_through_the_read_only_path():
    """With launch overlap the launch before may write q, k_new and v_new while the 8-bit decode is already resident, so none of
    its loads may promise that nobody writes (ld.global.nc, __ldg, __restrict__ pointers to const)."""
    for name in ("flux_decode_kvq.cu", "flux_decode_fused.cu", "flux_decode_common.h", "flux_kvq.h"):
        assert not re.search(r"__ldg\s*\(|ld\.global(\.\w+)*\.nc|__restrict__", _code(name)), name
