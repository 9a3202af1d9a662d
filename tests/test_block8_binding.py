"""The binding's checks of what block calls are given, on the host."""
from types import SimpleNamespace

import pytest
import torch

from paper_2112_05923_amd import podrollout as pr


def _on(device, dtype, *shape):
    """What the binding looks at of a contiguous tensor on a GPU."""
    return SimpleNamespace(is_cuda=True, dtype=dtype, shape=torch.Size(shape), device=torch.device(device), is_contiguous=lambda: True)


def test_codes_and_scales_are_on_one_device():
    codes = _on("cuda:0", torch.float8_e4m3fn, 4, 256)
    assert pr.Blocks8(codes, _on("cuda:0", torch.uint8, 4, 2), 200).shape == (4, 200)
    with pytest.raises(ValueError):
        pr.Blocks8(codes, _on("cuda:1", torch.uint8, 4, 2), 200)


def test_a_workspace_of_less_than_its_alignment_is_empty():
    room = torch.empty(1024, dtype=torch.uint8)
    for at in range(0, 512, 5):
        for n in (0, 3, 100, 400):
            part = room[at:at + n]
            p, left = pr._aligned_ptr(part)
            assert p % 256 == 0 and left >= 0 and (left == 0 or p + left == part.data_ptr() + n)
