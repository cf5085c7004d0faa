"""The Python side of the 8-bit cache without a GPU: its C struct is always that of its tensors."""
import numpy as np
import pytest
import torch

import paper_2607_02043_amd as mla


def tensors(n, P):
    return torch.zeros((n, P, 576), dtype=torch.uint8), torch.ones((n, P // 16, 2), dtype=torch.bfloat16)


def test_replaced_tensors():
    c = mla.LatentCache8(num_pages=3, page_size=32, device="cpu")
    first = c.c.data
    d, s = tensors(5, 64)
    c.data, c.scales = d, s
    assert (c.c.data, c.c.scales) == (d.data_ptr(), s.data_ptr()) and c.c.data != first
    assert (c.num_pages, c.page_size) == (5, 64)


@pytest.mark.parametrize("bad", [lambda d, s: (d[:, :, :512], s), (lambda d, s: (d, s[:2])), (lambda d, s: (d, s.float())),
                                 (lambda d, s: (d.to(torch.int16), s))])
def test_replaced_tensors_are_checked(bad):
    c = mla.LatentCache8(num_pages=3, page_size=32, device="cpu")
    c.data, c.scales = bad(*tensors(3, 32))
    b = mla.DeviceBatch([1], [3], np.zeros((1, 1)), 32, 3, device="cpu")
    with pytest.raises(ValueError, match="must be contiguous"):
        mla._cache8(b, c, -1)  # what every call goes through; -1: the device of these tensors
    with pytest.raises(ValueError, match="must be contiguous"):
        c.c


def test_a_tensor_that_moved():
    d, s = tensors(3, 32)
    c = mla.LatentCache8(data=d, scales=s)
    other = torch.zeros((3, 32, 576), dtype=torch.uint8)
    d.set_(other)
    assert c.c.data == other.data_ptr()
    d.set_(torch.zeros((2, 32, 576), dtype=torch.uint8))
    with pytest.raises(ValueError, match="scales"):
        c.c
