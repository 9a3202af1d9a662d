"""Layers on 8-bit blocks through the binding: in-place calls raise, columns of one buffer do not."""
import pytest
import torch

from paper_2112_05923_amd import podrollout as pr
from test_gpu_block8 import DEV, _layer

pytestmark = pytest.mark.gpu


def test_in_place_calls_raise_and_leave_everything_alone():
    x, w, b = _layer(None, 1500, 256, 256)
    weights, bias, xd = pr.Weights8(w.to(DEV)), b.to(DEV), x.to(DEV)
    h = pr.block8_quantize(xd)
    codes, scales = h.q.view(torch.uint8).clone(), h.scale.clone()
    for call in (lambda: pr.block8_linear(h, weights, bias, True, h), lambda: pr.block8_linear(xd, weights, bias, True, xd),
                 lambda: pr.block8_linear_grads(xd, h, weights, None, dx=xd),
                 lambda: pr.block8_linear(h, weights, bias, True, pr.Blocks8(h.q, torch.zeros_like(h.scale), 256))):
        with pytest.raises(pr.PodError) as e:
            call()
        assert e.value.code == pr.PR_EINVAL
    assert torch.equal(h.q.view(torch.uint8), codes) and torch.equal(h.scale, scales) and torch.equal(xd.cpu(), x)


def test_a_layer_between_columns_of_one_buffer():
    x, w, b = _layer(None, 700, 100, 60)
    weights, bias = pr.Weights8(w.to(DEV)), b.to(DEV)
    room = torch.zeros((700, 170), device=DEV)
    room[:, 5:105] = x.to(DEV)
    pr.block8_linear(room[:, 5:105], weights, bias, True, room[:, 105:165])
    assert torch.equal(room[:, 105:165], pr.block8_linear(x.to(DEV), weights, bias, True))
    assert torch.equal(room[:, 5:105].cpu(), x) and not room[:, :5].any() and not room[:, 165:].any()
