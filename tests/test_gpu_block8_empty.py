"""Gradients of no rows of layers on 8-bit blocks: every entry is written, where a launch does not reach them all too."""
import ctypes as C

import pytest
import torch

from paper_2112_05923_amd import podrollout as pr

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("agents,ins,outs", [(1, 70, 30), (3, 1000, 1200), (1, 33000, 33001)])
def test_gradients_of_no_rows_are_zero(agents, ins, outs):
    dev = torch.device("cuda:0")
    dW, db = torch.full((agents, ins, outs), 7.0, device=dev), torch.full((agents, outs), 7.0, device=dev)
    packed = torch.zeros(512, dtype=torch.uint8, device=dev)  # (of no rows nothing of the weights is read)
    layer = pr.PrBlock8Layer(agents, ins, outs, 0, 0)
    pr._b8_call("block8_linear_grads", dev, C.byref(layer), pr.PR_B8_F32, None, outs, None, None, None, None, pr._aligned_ptr(packed)[0],
                pr.PR_B8_F32, None, ins, dW.data_ptr(), db.data_ptr(), None, 0)
    assert int(torch.count_nonzero(dW)) == 0 and int(torch.count_nonzero(db)) == 0
