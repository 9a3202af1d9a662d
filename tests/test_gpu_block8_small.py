"""Layers on 8-bit blocks whose sums are small: results keep their relative precision down to the smallest, in every kernel.

Every row has one input that is not zero, so a sum is one product of two codes, exact in any arithmetic, and what is seen is the
activation and the rounding of its result.  Rows are of every magnitude from 1e-12 to 10, and a few of 1e-30.  Oracle and
roundings as in test_gpu_block8.
"""
import pytest
import torch

import block8_oracle as o
from paper_2112_05923_amd import podrollout as pr
from test_gpu_block8 import DEV, TYPES, _within

pytestmark = pytest.mark.gpu

# rows, ins, outs, source: few rows; weights resident (one, three blocks of inputs; a head); in tiles; plain rows a workgroup of
# one and of several blocks of features; and what the others do not take
CASES = [(48, 301, 200, "blocks"), (100, 40, 130, "bf16"), (1500, 100, 100, "blocks"), (1500, 300, 120, "blocks"), (1500, 500, 30, "blocks"),
         (1500, 640, 200, "blocks"), (1500, 301, 128, "f32"), (33100, 40, 256, "f32"), (33100, 40, 260, "bf16"), (1500, 5, 130, "f32")]


def _case(rows, ins, outs):
    gen = torch.Generator().manual_seed(rows + ins + outs)
    size = torch.pow(10.0, torch.rand(rows, generator=gen, dtype=torch.float64) * 13 - 12)
    size[::97] = 1e-30
    x = torch.zeros(rows, ins)
    x[torch.arange(rows), torch.arange(rows) % ins] = (size * (1 - 2 * torch.randint(0, 2, (rows,), generator=gen))).float()
    w = (0.1 + torch.rand((ins, outs), generator=gen)) * (1 - 2 * torch.randint(0, 2, (ins, outs), generator=gen))
    return x, w


@pytest.mark.parametrize("rows,ins,outs,source", CASES)
def test_tanh_of_small_sums(rows, ins, outs, source):
    x, w = _case(rows, ins, outs)
    x = x.to(TYPES.get(source, torch.float32))
    z = o.values(x) @ o.weight_values(w)
    y = torch.tanh(z)
    xin = pr.block8_quantize(x.to(DEV)) if source == "blocks" else x.to(DEV)
    weights = pr.Weights8(w.to(DEV))
    # fp32: the function to a few 2^-24 of its value below 1/4, 2^-22 absolute above (1e-6 of a value of at least .24)
    _within(pr.block8_linear(xin, weights, None, True), y, (1e-6 + 2.0 ** -24) * y.abs(), "f32")
    # bf16: z itself where z^2 / 3 is below 2.1e-5, and 2^-22 absolute above (3.1e-5 of 2^-7)
    _within(pr.block8_linear(xin, weights, None, True, torch.bfloat16), y, (3.1e-5 + 2.0 ** -8 * (1 + 3.1e-5)) * y.abs(), "bf16")
    # blocks: to 1e-5 of the value where no sum of the block reaches 1/2, 2^-22 absolute in the others
    out = pr.block8_linear(xin, weights, None, True, "blocks")
    most = o.pad(z.abs()).unflatten(-1, (-1, o.BLOCK)).amax(-1)
    err = torch.where((most >= 0.49).repeat_interleave(o.BLOCK, -1)[..., :outs], 2.0 ** -22 + 1e-5 * y.abs(), 1e-5 * y.abs())
    amount = lambda v: o.pad(v.clamp(min=0.0)).unflatten(-1, (-1, o.BLOCK)).amax(-1)
    low, high = o.exponents(amount(y.abs() - err)), o.exponents(amount(y.abs() + err))
    e = out.scale.to(torch.int64).cpu() - 127
    assert bool(((e >= low) & (e <= high)).all())
    unit = o.power(high).repeat_interleave(o.BLOCK, -1)[..., :outs]
    _within(pr.block8_dequantize(out, torch.float32), y, err + 2.0 ** -4 * (y.abs() + err) + 2.0 ** -10 * unit, "blocks")


@pytest.mark.parametrize("rows", [48, 1500])
def test_maxima_just_above_a_border_of_the_rule(rows):
    """Blocks whose largest sum is 1.5e-6 to 2e-6 in steps of half a per cent, of either sign: every value is finite, and within
    half a step of its code."""
    x = torch.zeros(rows, 64)
    x[:, 0] = 2.0 ** -19 * (0.75 + 0.005 * (torch.arange(rows) % 60).float())
    w = torch.zeros(64, 128)
    w[0] = torch.where(torch.arange(128) % 2 == 0, 1.0, -1.0) * (1 - 0.001 * torch.arange(128).float())
    bias = x[0, 0] * 0.001 * torch.arange(128).float()
    z = o.values(x) @ o.weight_values(w) + bias.double()
    y = torch.tanh(z)
    got = pr.block8_dequantize(pr.block8_linear(pr.block8_quantize(x.to(DEV)), pr.Weights8(w.to(DEV)), bias.to(DEV), True, "blocks"),
                               torch.float32)
    err = o.sum_bound(o.values(x), o.weight_values(w), bias) + 1e-5 * y.abs()
    unit = o.power(o.exponents((y.abs() + err).amax(-1)))[:, None]
    _within(got, y, err + 2.0 ** -4 * (y.abs() + err) + 2.0 ** -10 * unit)
