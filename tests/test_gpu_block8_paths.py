"""Every way that layers on 8-bit blocks are computed, held to exact results over all of their rows.

Entries are small whole numbers, and weights of layers 64ths of them: what is stored is stored exactly, and all sums are exact in
fp32, so sums, gradients and their rounded forms have to be equal bit for bit, and an activation is seen by itself.  Blocks have
scales of their own, a few powers of two apart.  The sizes are those at which the rules of the launches choose each kernel (test_block8_launches holds the tables to that): rows by the ten thousand,
that leave a ragged tile behind, workgroups that walk several blocks, wavefronts without a block of their own, rows far apart.
"""
import pytest
import torch

import block8_oracle as o
from paper_2112_05923_amd import podrollout as pr
from test_gpu_block8 import DEV, TYPES

pytestmark = pytest.mark.gpu

# agents, rows, ins, outs
PLAIN = [(None, 33000, 301, 140), (None, 33000, 301, 300), (None, 33100, 40, 512), (None, 17000, 70, 300), (3, 11001, 130, 257), (None, 1500, 5, 130),
         (None, 130, 301, 128), (2, 700, 1000, 100), (None, 4000, 200, 600)]
STORED = [(None, 1500, 100, 30), (None, 1500, 100, 9), (None, 1500, 200, 30), (None, 1500, 200, 9), (None, 1500, 300, 30), (None, 1500, 300, 9),
          (None, 1500, 500, 30), (None, 1500, 500, 9), (None, 70000, 500, 129), (None, 65800, 130, 140), (None, 140000, 128, 96), (None, 3001, 1100, 520),
          (20, 1300, 640, 200), (None, 90, 700, 300)]
GRADS = [(None, 17000, 301, 130), (None, 17000, 512, 256), (None, 33000, 512, 512), (None, 33001, 400, 512), (None, 33000, 384, 30), (None, 33000, 300, 200),
         (None, 17000, 300, 900), (None, 1300, 300, 900), (None, 17100, 257, 1024), (None, 300, 200, 1100), (None, 1700, 130, 2000), (70, 200, 600, 300),
         (None, 9000, 300, 32), (None, 66000, 200, 70), (3, 12000, 512, 512), (None, 100, 300, 128)]


def whole(shape, most, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=gen, device=DEV).float()


def scales(shape, most, seed, rows=1):
    """Powers of two up to 2^most and down to 2^-most for each `rows` rows x 128 columns."""
    lead, (n, cols) = shape[:-2], shape[-2:]
    e = whole(lead + ((n + rows - 1) // rows, (cols + o.BLOCK - 1) // o.BLOCK), most, seed)
    return o.power(e).float().repeat_interleave(rows, -2)[..., :n, :].repeat_interleave(o.BLOCK, -1)[..., :cols]


def product(a, b):
    """In 64 bits, agent by agent."""
    a, b = a.double(), b.double()
    return a @ b if a.dim() == 2 else torch.stack([p @ q for p, q in zip(a, b)])


def _same(got, want, what):
    assert got.shape == want.shape and torch.equal(got, want), (what, int((got != want).sum()), (got != want).nonzero()[:3].tolist())


def _near(got, want, bound, what):
    off = (got.double() - want).abs() - bound
    assert got.shape == want.shape and bool((off <= 0).all()), (what, float(off.max()), (~(off <= 0)).nonzero()[:3].tolist())


def _check_layer(xin, x, weights, w, b):
    """To every kind of result, with and without tanh."""
    outs = w.shape[-1]
    z = product(x, w) + b.double()[..., None, :]
    for kind in TYPES.values():
        _same(pr.block8_linear(xin, weights, b, False, kind), z.float().to(kind), kind)
    got, want = pr.block8_linear(xin, weights, b, False, "blocks"), pr.block8_quantize(z.float())
    _same(got.scale, want.scale, "scale bytes")
    _same(got.q.float(), want.q.float(), "codes")
    y = torch.tanh(z)
    _near(pr.block8_linear(xin, weights, b, True), y, (1e-6 + 2.0 ** -24) * y.abs(), "tanh f32")
    _near(pr.block8_linear(xin, weights, b, True, torch.bfloat16), y, (3.1e-5 + 2.0 ** -8 * (1 + 3.1e-5)) * y.abs(), "tanh bf16")
    err = 2.0 ** -22 + 1e-5 * y.abs()
    unit = o.power(o.exponents(o.pad(y.abs() + err).unflatten(-1, (-1, o.BLOCK)).amax(-1))).repeat_interleave(o.BLOCK, -1)[..., :outs]
    _near(pr.block8_dequantize(pr.block8_linear(xin, weights, b, True, "blocks"), torch.float32), y,
          err + 2.0 ** -4 * (y.abs() + err) + 2.0 ** -10 * unit, "tanh blocks")


def _layer(agents, rows, ins, outs):
    lead = () if agents is None else (agents,)
    sx, sw = lead + (rows, ins), lead + (ins, outs)
    return (whole(sx, 2, rows + ins) * scales(sx, 2, 1), whole(sw, 2, outs) * scales(sw, 2, 2, o.BLOCK) / 64, whole(lead + (outs,), 64, 3) / 64)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", PLAIN)
def test_products_of_plain_rows(shape, kind):
    x, w, b = _layer(*shape)
    _check_layer(x.to(TYPES[kind]), x, pr.Weights8(w), w, b)


@pytest.mark.parametrize("shape", STORED)
def test_products_of_blocks(shape):
    x, w, b = _layer(*shape)
    _check_layer(pr.block8_quantize(x), x, pr.Weights8(w), w, b)


def _case(agents, rows, ins, outs, tanh):
    lead = () if agents is None else (agents,)
    sx, sw, sy = lead + (rows, ins), lead + (ins, outs), lead + (rows, outs)
    x, w, dy = whole(sx, 2, rows) * scales(sx, 1, 1), whole(sw, 2, outs) * scales(sw, 3, 2, o.BLOCK), whole(sy, 3, ins)
    y = whole(sy, 2, rows + 1) / 4 * scales(sy, 1, 3).clamp(min=1.0) if tanh else None  # up to 1/2, or to 1
    g = dy if y is None else dy * (1 - y * y)
    turned = lambda t: t.transpose(-1, -2).contiguous()
    return x, w, dy, y, product(g, turned(w)), product(turned(x), g).float(), g.double().sum(-2).float()


@pytest.mark.parametrize("tanh", [True, False])
@pytest.mark.parametrize("shape", GRADS)
def test_gradients(shape, tanh):
    x, w, dy, y, dx, dW, db = _case(*shape, tanh)
    weights, xb, yb = pr.Weights8(w), pr.block8_quantize(x), None if y is None else pr.block8_quantize(y)
    for kind in TYPES.values():
        for dkind in (*TYPES.values(), None):
            got = pr.block8_linear_grads(dy.to(kind), xb, weights, yb, dx=dkind)
            _same(got[1], dW, ("dW", kind, dkind))
            _same(got[2], db, ("db", kind, dkind))
            assert dkind is not None or got[0] is None
            if dkind is not None:
                _same(got[0], dx.float().to(dkind), ("dx", kind, dkind))


FAR_ROWS, FAR_BYTES = 1030, 1 << 26  # 32 rows are 2 GiB apart


def _far(room, kind, cols, at):
    """Rows in a buffer of 69 GB, `at` elements behind their places."""
    t = room.view(kind)
    return t.as_strided((FAR_ROWS, cols), (FAR_BYTES // t.element_size(), 1), at)


@pytest.fixture(scope="module")
def room():
    t = torch.empty(FAR_ROWS * FAR_BYTES, dtype=torch.uint8, device=DEV)  # (none of it but the rows is touched)
    yield t
    del t
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", TYPES)
def test_rows_far_apart(room, kind):
    t, ins, outs = TYPES[kind], 200, 300
    x, w, b = _layer(None, FAR_ROWS, ins, outs)
    weights, z = pr.Weights8(w), product(x, w) + b.double()
    far_x, far_y = _far(room, t, ins, 3), _far(room, t, outs, 1001)
    far_x.copy_(x)
    for xin in (far_x, x.to(t), pr.block8_quantize(far_x)):
        far_y.zero_()
        pr.block8_linear(xin, weights, b, False, far_y)
        _same(far_y, z.float().to(t), "y")
    _same(pr.block8_linear(far_x, weights, b, False, t), z.float().to(t), "y of far rows")
    _same(pr.block8_dequantize(pr.block8_linear(far_x, weights, b, False, "blocks"), out=far_y),
          pr.block8_dequantize(pr.block8_quantize(z.float()), t), "blocks")
    for tanh in (True, False):
        x, w, dy, y, dx, dW, db = _case(None, FAR_ROWS, ins, outs, tanh)
        far_dy, far_dx = _far(room, t, outs, 7), _far(room, t, ins, 2001)
        far_dy.copy_(dy)
        far_dx.zero_()
        got = pr.block8_linear_grads(far_dy, pr.block8_quantize(x), pr.Weights8(w), None if y is None else pr.block8_quantize(y), dx=far_dx)
        _same(far_dx, dx.float().to(t), "dx")
        _same(got[1], dW, "dW")
        _same(got[2], db, "db")


@pytest.mark.parametrize("of_rows,of_weights", [(100, -103), (-100, 97), (55, 50), (-55, -50)])
@pytest.mark.parametrize("shape", [(48, 300, 200), (1500, 300, 30), (3001, 640, 200), (1500, 5, 130)])
def test_scales_at_the_far_ends(shape, of_rows, of_weights):
    """Rows and weights whose scales are far from 1, up and down, with products and gradients of either size."""
    x, w, b = _layer(None, *shape)
    dy = whole((shape[0], shape[2]), 3, 5)
    x, w, b = x * 2.0 ** of_rows, w * 2.0 ** of_weights, b * 2.0 ** (of_rows + of_weights)
    weights, xb, z = pr.Weights8(w), pr.block8_quantize(x), product(x, w) + b.double()
    for xin in (x, xb):
        for kind in TYPES.values():
            _same(pr.block8_linear(xin, weights, b, False, kind), z.float().to(kind), kind)
        got, want = pr.block8_linear(xin, weights, b, False, "blocks"), pr.block8_quantize(z.float())
        _same(got.scale, want.scale, "scale bytes")
        _same(got.q.float(), want.q.float(), "codes")
    dx, dW, db = pr.block8_linear_grads(dy, xb, weights, dx=torch.float32)
    _same(dx, product(dy, w.T.contiguous()).float(), "dx")
    _same(dW, product(x.T.contiguous(), dy).float(), "dW")
    _same(db, dy.double().sum(0).float(), "db")
