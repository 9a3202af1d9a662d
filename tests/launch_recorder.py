"""Which kernels a call of the C ABI launches, and how: the library in a process of its own whose HIP runtime (launch_recorder.c)
prints launches instead of making them.  No device is touched; pointers are numbers.

    record([("block8_quantize", [0, 4, 10, 0, A, 10, B, C])]) -> [Call(code, [Launch(kernel, grid, block, lds)])]

A list among the arguments is a block layer (agents, in, out, tanh, rows), "out" room for a number that comes back.
"""
import collections
import ctypes as C
import json
import os
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2112_05923_amd", "libpodrollout.so")
Launch = collections.namedtuple("Launch", "kernel grid block lds")
Call = collections.namedtuple("Call", "code launches out")


def _lines(calls, env):
    with tempfile.TemporaryDirectory() as room:
        runtime = os.path.join(room, "recorder.so")
        subprocess.run(["gcc", "-std=gnu11", "-O1", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "launch_recorder.c"), "-o", runtime], check=True)
        r = subprocess.run([sys.executable, os.path.abspath(__file__), runtime], input=json.dumps(calls), capture_output=True, text=True,
                           timeout=300, env=dict(os.environ, **env))
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout.splitlines()


def _readable(names):
    out = subprocess.run(["c++filt"], input="\n".join(names), capture_output=True, text=True).stdout.split("\n")
    return [n.replace("void ", "").replace("pod::b8::(anonymous namespace)::", "").split("(")[0] for n in out[:len(names)]]


def kernels():
    """All kernels of the library."""
    return _readable([l.split()[1] for l in _lines([], {"RECORDER_LISTS_KERNELS": "1"}) if l.startswith("kernel ")])


def record(calls, **env):
    got, launches = [], []
    for line in _lines(calls, env):
        word, *rest = line.split()
        if word == "launch":
            n = [int(v) for v in rest[1:]]
            launches.append(Launch(rest[0], tuple(n[:3]), tuple(n[3:6]), n[6]))
        elif word == "call":
            got.append(Call(int(rest[0]), launches, int(rest[1])))
            launches = []
    names = iter(_readable([l.kernel for c in got for l in c.launches]))
    return [Call(c.code, [l._replace(kernel=next(names)) for l in c.launches], c.out) for c in got]


class _Layer(C.Structure):
    _fields_ = [("n_agents", C.c_int32), ("in_dim", C.c_int32), ("out_dim", C.c_int32), ("tanh", C.c_int32), ("rows", C.c_int64)]


def _run(runtime):
    C.CDLL(runtime, mode=C.RTLD_GLOBAL)
    l = C.CDLL(LIB)
    for name, args in json.load(sys.stdin):
        out, keep, given = C.c_size_t(0), [], []
        for a in args:
            if isinstance(a, list):
                keep.append(_Layer(*a))
                given.append(C.byref(keep[-1]))
            elif a == "out":
                given.append(C.byref(out))
            else:
                given.append(None if a is None else C.c_int64(a))
        code = getattr(l, name)(*given)
        C.CDLL(None).fflush(None)
        print("call", code, out.value, flush=True)


if __name__ == "__main__":
    _run(sys.argv[1])
