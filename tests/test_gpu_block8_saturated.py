"""Where 8-bit checkpoints of a layer's outputs cut gradients off: |tanh z| from 31/32 on, as the header says, and not before; and
the way around it."""
import math

import pytest
import torch

import block8_oracle as o
from paper_2112_05923_amd import podrollout as pr
from test_gpu_block8 import DEV, _within

pytestmark = pytest.mark.gpu


def test_units_from_31_32_on_have_no_gradient_from_blocks_but_from_plain_outputs():
    border = math.atanh(31 / 32)
    z = torch.cat([torch.linspace(0.0, border - 1e-3, 60), torch.linspace(border + 1e-3, 4.0, 60)])
    x, w = torch.ones(40, 8, device=DEV), torch.zeros(8, 120, device=DEV)
    weights = pr.Weights8(w)
    xb, dy = pr.block8_quantize(x), torch.ones(40, 120, device=DEV)
    blocks = pr.block8_linear(xb, weights, z.to(DEV), True, "blocks")
    plain = pr.block8_linear(xb, weights, z.to(DEV), True)
    _, dW, db = pr.block8_linear_grads(dy, xb, weights, blocks)
    assert bool((db[:60] > 0).all()) and not db[60:].any() and not dW[:, 60:].any()
    _, dW, db = pr.block8_linear_grads(dy * (1.0 - plain * plain), xb, weights)
    # each row's g is rounded to bf16 once; 1 - y^2 of an fp32 tanh is off by 2e-6; forty equal rows add up exactly enough
    want = 1.0 - torch.tanh(z.double()) ** 2
    _within(db, 40 * want, 40 * (want * 2.0 ** -8 + 4e-6) + 42 * 2.0 ** -23 * 40 * want)
    _within(dW, (40 * want).expand(8, -1), (40 * (want * 2.0 ** -8 + 4e-6) + 42 * 2.0 ** -23 * 40 * want).expand(8, -1))
    assert float(db.min()) > 0


def test_factors_are_as_far_off_as_the_codes():
    y = torch.linspace(-1, 1, 4001)[:, None].expand(-1, 4).contiguous()
    stored = o.values(y)
    got = pr.block8_linear_grads(torch.ones(4001, 4, device=DEV), pr.block8_quantize(torch.eye(4001)[:, :1].to(DEV)),
                                 pr.Weights8(torch.ones(1, 4, device=DEV)), pr.block8_quantize(y.to(DEV)), dx=torch.float32)[0]
    exact = 4 * (1.0 - stored[:, :1] ** 2)
    _within(got, exact, exact * 2.0 ** -8 + 1e-6)
    assert float((exact / 4 - (1.0 - y[:, :1].double() ** 2)).abs().max()) <= 1 / 16
