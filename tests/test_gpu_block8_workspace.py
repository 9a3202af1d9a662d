"""One workspace for many rows, used for fewer: the same gradients, and nothing written behind it or with too little of it."""
import pytest
import torch

from paper_2112_05923_amd import podrollout as pr
from test_gpu_block8 import DEV, _layer, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("agents,ins,outs,most", [(None, 300, 200, 9000), (None, 130, 33, 5000), (None, 512, 30, 3000), (3, 70, 40, 700), (70, 300, 260, 200)])
def test_a_workspace_of_many_rows_serves_fewer(agents, ins, outs, most):
    x, w, _ = _layer(agents, most, ins, outs, seed=7)
    weights, dy = pr.Weights8(w.to(DEV)), _rand(x.shape[:-1] + (outs,), 8).to(DEV)
    given = pr.block8_workspace(weights, most, DEV)
    size = given.numel() - 256  # (and what aligns it)
    room = torch.full((size + 8192,), 37, dtype=torch.uint8, device=DEV)
    at = -room.data_ptr() % 256
    for rows in (most, most - 1, most // 2 + 1, most // 7, 128, 5):
        xb, d = pr.block8_quantize(x[..., :rows, :].contiguous().to(DEV)), dy[..., :rows, :].contiguous()
        want = pr.block8_linear_grads(d, xb, weights)
        got = pr.block8_linear_grads(d, xb, weights, workspace=room[at:at + size])
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
        assert bool((room[at + size:] == 37).all()) and bool((room[:at] == 37).all())


def test_too_little_of_it_is_refused():
    x, w, _ = _layer(None, 2000, 300, 200, seed=7)
    weights, xb, dy = pr.Weights8(w.to(DEV)), pr.block8_quantize(x.to(DEV)), _rand((2000, 200), 8).to(DEV)
    with pytest.raises(pr.PodError) as e:
        pr.block8_linear_grads(dy, xb, weights, workspace=pr.block8_workspace(weights, 200, DEV))
    assert e.value.code == pr.PR_ENOMEM


def test_one_that_is_not_there_is_refused():
    """A byte that stands for many, and the few bytes in front of a boundary."""
    x, w, _ = _layer(None, 2000, 300, 200, seed=7)
    weights, xb, dy = pr.Weights8(w.to(DEV)), pr.block8_quantize(x.to(DEV)), _rand((2000, 200), 8).to(DEV)
    need = pr.block8_workspace(weights, 2000, DEV).numel()
    with pytest.raises(TypeError):
        pr.block8_linear_grads(dy, xb, weights, workspace=torch.zeros(1, dtype=torch.uint8, device=DEV).expand(need))
    short = torch.zeros(512, dtype=torch.uint8, device=DEV)
    with pytest.raises(pr.PodError) as e:
        pr.block8_linear_grads(dy, xb, weights, workspace=short[1:9])
    assert e.value.code == pr.PR_ENOMEM
