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


def _kernels(text):
    """Text from each __global__ to the next (helpers between two kernels belong to the one before)."""
    parts = re.split(r"(?=__global__)", text)
    return parts


@pytest.mark.parametrize("name", sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "*.cu"))))
def test_no_kernel_lets_the_next_one_start_before_its_own_wait(name):
    """A decode with launch overlap reads cache blocks and tables that the launch directly before it does not write, and counts on every
    earlier launch being done.  That holds only if the launch before passes on the permission to start after its own wait: given earlier,
    the decode could run beside a store, or a router, two launches back."""
    for part in _kernels(_code(name)):
        marks = [m.group(1) for m in re.finditer(r"griddepcontrol\.(wait|launch_dependents)", part)]
        for i, mark in enumerate(marks):
            assert mark == "wait" or (i > 0 and marks[i - 1] == "wait"), (name, part[:80], marks)
        # where the two are wrapped in functions of a kernel's own
        calls = [m.group(1) for m in re.finditer(r"\b(wait|release)\(\);", part)]
        for i, call in enumerate(calls):
            assert call == "wait" or (i > 0 and calls[i - 1] == "wait"), (name, calls)
