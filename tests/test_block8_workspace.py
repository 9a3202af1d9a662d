"""Workspace of the block layers' gradients, on the host: one that serves many rows serves fewer, and none is asked for that
nothing is put into."""
import ctypes as C
import shutil

import pytest

from paper_2112_05923_amd import podrollout as pr
from test_block8_launches import grads

SIZES = [(1, 512, 512), (1, 128, 512), (1, 129, 33), (1, 1024, 1024), (1, 512, 30), (1, 301, 512), (3, 700, 300), (64, 301, 256), (64, 64, 64),
         (1, 1, 1), (7, 3001, 1024)]


def _bytes(agents, ins, outs, rows):
    n = C.c_size_t(0)
    assert pr.lib().block8_workspace_bytes(C.byref(pr.PrBlock8Layer(agents, ins, outs, 1, rows)), C.byref(n)) == pr.PR_OK
    return n.value


ROWS = sorted(set(list(range(1, 40)) + [128 * k + d for k in range(1, 90) for d in (-1, 0, 1, 33)] + [2 ** k + d for k in range(7, 21) for d in (-1, 0, 1)]))


@pytest.mark.parametrize("agents,ins,outs", SIZES)
def test_more_rows_never_ask_for_less(agents, ins, outs):
    sizes = [_bytes(agents, ins, outs, r) for r in ROWS]
    assert sizes == sorted(sizes)
    assert sizes[0] > 0 and sizes[-1] <= 513 * agents * (ins + 1) * outs * 4
    assert _bytes(agents, ins, outs, 0) == 0


@pytest.mark.skipif(shutil.which("gcc") is None or shutil.which("c++filt") is None, reason="no gcc")
def test_a_workspace_of_many_rows_serves_any_fewer():
    from launch_recorder import record
    calls = []
    for agents, ins, outs in SIZES:
        for most in (8192, 4096, 100000, 16000):
            room = _bytes(agents, ins, outs, most)
            for rows in [r for r in ROWS if r <= most][::3] + [most // 2, most - 1, most]:
                name, args = grads(rows, ins, outs, agents=agents)
                calls.append((name, args[:-1] + [room]))
    for call, got in zip(calls, record(calls)):
        assert got.code == pr.PR_OK, call


def test_results_of_one_run_need_no_copy_of_them():
    for agents, ins, outs, rows in ((64, 1024, 1024, 1000), (1, 512, 512, 100), (1, 8192, 8192, 100000)):
        assert _bytes(agents, ins, outs, rows) < 4096
