"""Layouts that the calls on packed rows take, without a device."""
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
