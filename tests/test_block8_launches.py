"""What calls of the 8-bit block layers launch, seen by a process whose HIP runtime only records (launch_recorder)."""
import shutil

import pytest

from launch_recorder import kernels, record
from paper_2112_05923_amd import podrollout as pr

pytestmark = pytest.mark.skipif(shutil.which("gcc") is None or shutil.which("c++filt") is None, reason="no gcc")

F32, BF16, BLOCKS = pr.PR_B8_F32, pr.PR_B8_BF16, pr.PR_B8_BLOCKS
X, XS, W, B, Y, YS, DY, DX, DW, DB, WS = ((i + 1) << 44 for i in range(11))  # places far apart that no call touches


def linear(rows, ins, outs, x=BLOCKS, y=BLOCKS, agents=1, ldx=None, ldy=None):
    return ("block8_linear", [0, [agents, ins, outs, 1, rows], x, X, XS, ldx or ins, W, B, y, Y, YS, ldy or outs])


def grads(rows, ins, outs, dy=BF16, dx=BF16, tanh=1, agents=1):
    y = (Y, YS) if tanh else (None, None)
    return ("block8_linear_grads", [0, [agents, ins, outs, tanh, rows], dy, DY, outs, *y, X, XS, W, dx, DX, ins, DW, DB, WS, 1 << 43])


def test_an_error_of_the_runtime_reaches_the_caller():
    """The resident kernels ask for more LDS than a kernel has by itself; where that is refused the call has not run."""
    calls = [linear(262144, 512, 512), linear(262144, 512, 30, y=F32), linear(70000, 100, 60, y=BF16)]
    for c in record(calls):
        assert c.code == pr.PR_OK and [l.kernel.split("<")[0] for l in c.launches] == ["linear_resident_kernel"]
    for c in record(calls, RECORDER_REFUSES_ATTRIBUTES="1"):
        assert c.code == pr.PR_EHIP and not c.launches


# (what such a call reads and writes is up to 300 GB: the largest cards hold the first four)
WIDEST = [linear(1 << 30, 8, 256, x=BF16), linear(1 << 30, 8, 129, x=BF16, y=BF16), linear(1 << 29, 8, 257, x=BF16, y=BF16),
          linear(1 << 29, 8, 512, x=BF16), linear(1 << 30, 5, 128, x=BF16), linear(1 << 30, 8, 128, x=BF16), linear(1 << 30, 128, 128),
          grads(1 << 30, 128, 8), grads(1 << 30, 64, 64, tanh=0), grads(1000, 65536, 65536), grads(100, 1 << 20, 1 << 15)]


def test_the_longest_calls_stay_within_a_launch():
    for call, got in zip(WIDEST, record(WIDEST)):
        assert got.code == pr.PR_OK and got.launches, (call, got)


def test_gradients_of_no_rows_are_zeroed_whole():
    """dW of 2^32 entries too: the launches' threads cover it, and db once."""
    for agents, ins, outs in ((1, 65536, 65536), (64, 8192, 8192), (1, 70, 30), (3, 20000, 20000)):
        got, = record([grads(0, ins, outs, agents=agents)])
        assert got.code == pr.PR_OK
        entries = agents * (ins + 1) * outs
        splits = {"join_kernel<1>": 1, "join_kernel<4>": 4, "join_kernel<16>": 16}
        assert sum(l.grid[0] * l.block[0] // splits[l.kernel] for l in got.launches) >= entries


def test_the_gpu_tests_reach_every_kernel():
    """The sizes of the tests on a GPU, by the rules of the launches, against the kernels that the library has."""
    import test_gpu_block8_paths as paths
    import test_gpu_block8_small as small
    kinds = {"f32": F32, "bf16": BF16, "blocks": BLOCKS}
    plain = (F32, BF16)
    calls = [("block8_quantize", [0, 4, 10, k, X, 10, Y, YS]) for k in plain] + [("block8_dequantize", [0, 4, 10, Y, YS, k, X, 10]) for k in plain]
    calls.append(("block8_pack_weights", [0, [1, 10, 10, 0, 0], W, Y, 1 << 30]))
    calls += [linear(*s[:3], kinds[s[3]], y) for s in small.CASES for y in kinds.values()]
    calls += [linear(*s[1:], x, y, agents=s[0] or 1) for s in paths.PLAIN for x in plain for y in kinds.values()]
    calls += [linear(*s[1:], BLOCKS, y, agents=s[0] or 1) for s in paths.STORED for y in kinds.values()]
    calls += [grads(*s[1:], dy, dx, t, agents=s[0] or 1) for s in paths.GRADS for dy in plain for dx in plain for t in (0, 1)]
    far = {F32: paths.FAR_BYTES // 4, BF16: paths.FAR_BYTES // 2}
    calls += [linear(paths.FAR_ROWS, 200, 300, x, y, ldx=far.get(x), ldy=far[y]) for x in kinds.values() for y in plain]
    calls += [(n, [*a[:15], far[k], *a[16:]]) for k in plain for n, a in [grads(paths.FAR_ROWS, 200, 300, k, k)]]
    got = record(calls)
    assert all(c.code == pr.PR_OK for c in got), [(a, c) for a, c in zip(calls, got) if c.code != pr.PR_OK][:3]
    used = {l.kernel for c in got for l in c.launches}
    mine = {k for k in kernels() if k.startswith(("block8_", "linear_", "input_grads_", "weight_grads_", "join_kernel"))}
    assert used <= mine and not mine - used, sorted(mine - used)
