"""Layouts that the calls on packed rows take, without a device."""
import numpy as np
import pytest
import torch

from paper_2604_07394_b200 import flux


def test_one_head_may_have_any_head_stride():
    """With one head its stride says nothing: a contiguous tensor that torch shows with another one is as good as any."""
    x = torch.zeros(1, 5, 128, dtype=torch.bfloat16).transpose(0, 1)            # [5][1][128], strides (128, 640, 1)
    assert x.is_contiguous() and x.stride() == (128, 640, 1)
    assert flux._rows(x, 1, "k") == 128
    wide = torch.zeros(5, 512, dtype=torch.bfloat16)[:, 128:256].unsqueeze(1)
    assert flux._rows(wide, 1, "k") == 512
    lone = torch.zeros(3, 1, 128, dtype=torch.bfloat16)[1:2].transpose(0, 1).transpose(0, 1)
    assert flux._rows(lone, 1, "k") == 128
    for bad in (x[:, :, ::2], torch.zeros(128, 1, 5, dtype=torch.bfloat16).permute(2, 1, 0), x.transpose(0, 1)):
        with pytest.raises(ValueError):
            flux._rows(bad, 1, "k")
    # with more heads it has to be the row length
    with pytest.raises(ValueError):
        flux._rows(torch.zeros(2, 5, 128, dtype=torch.bfloat16).transpose(0, 1), 2, "k")


def test_row_bounds_are_whole_numbers_of_31_bits():
    """Bounds are never cut down to 32 bits or rounded on the way to the call."""
    for ok in ([0, 3, 9], (0, 3, 9), np.array([0, 3, 9]), np.array([0, 3, 9], dtype=np.uint8), torch.tensor([0, 3, 9]), [-1, 3, 9]):
        got = flux._bounds(ok, "q_rows")
        assert got.dtype == np.int32 and got.flags.c_contiguous and got.tolist() == [int(x) for x in ok]
    assert flux._bounds(np.arange(6, dtype=np.int32)[::2], "q_rows").tolist() == [0, 2, 4]
    for bad in ([0, 2 ** 32 + 5], [0, 2 ** 31], np.array([-2 ** 40, 0]), [0.0, 3.5], np.array([0.0, 3.0]), [False, True], np.array([0, 2 ** 63], dtype=np.uint64)):
        with pytest.raises(ValueError, match="q_rows"):
            flux._bounds(bad, "q_rows")
