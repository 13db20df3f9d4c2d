"""The gradients' norm keeps its partial sums within the workspace, whatever the list: the launches of a
call, recorded without a GPU."""
import ctypes
import json
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2607_24953_amd", "libq2d.so")

# (number of tensors, elements of each): many small ones, large ones among small ones, empty ones
LISTS = [[(1, 1)], [(10000, 12)], [(241, 1)], [(100000, 1)], [(5000, 2049)], [(3, 10 ** 9), (20000, 5)], [(1000, 16385)],
         [(700, 0), (300, 7), (5000, 0), (600, 2048)], [(20000, 40000)], [(1, 2 ** 40)], [(2000, 10 ** 7)]]


def test_parts_fit_the_workspace(tmp_path):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not found")
    so = os.path.join(str(tmp_path), "launch_recorder.so")
    subprocess.run(["gcc", "-std=c99", "-O1", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(HERE, "launch_recorder.c")], check=True)
    run = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(LISTS), capture_output=True, text=True,
                         timeout=300)
    assert run.returncode == 0, run.stderr[-4000:]
    for what, (size, norm, clip) in zip(LISTS, json.loads(run.stdout)):
        total = sum(n for n, e in what if e)
        for launches in (norm, clip):
            squares = [g for name, g in launches if "grad_square" in name]
            assert len(squares) <= total // 240 + 1 and min(squares) >= 1
            assert 8 * sum(squares) <= size, (what, sum(squares), size)
        # every other launch: the norm, and the scaling of 160 tensors at a time
        assert len(norm) == len(squares) + 1 and len(clip) == len(squares) + (total + 159) // 160


def _main(so):
    class Launch(ctypes.Structure):
        _fields_ = [("name", ctypes.c_char_p), ("grid", ctypes.c_uint32), ("block", ctypes.c_uint32), ("lds", ctypes.c_uint64)]
    rec = ctypes.CDLL(so, mode=ctypes.RTLD_GLOBAL)
    rec.recorded_launch.restype = ctypes.POINTER(Launch)
    lib = ctypes.CDLL(LIB)
    lib.q2d_grad_workspace.restype = ctypes.c_int64
    P, out = ctypes.c_void_p, []
    for what in json.load(sys.stdin):
        counts, data, at = [], [], 1 << 32
        for n, e in what:
            for _ in range(n):
                counts.append(e)
                data.append(at)
                at += 4 * e
        n = len(counts)
        args = ((P * n)(*data), (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*([0] * n)))
        size = lib.q2d_grad_workspace(n)
        got = [size]
        for clip in (False, True):
            rec.record_clear()
            if clip:
                s = lib.q2d_clip_grads(n, args[0], None, args[1], args[2], ctypes.c_double(1.0), None, P(1 << 20), P(1 << 21),
                                       ctypes.c_int64(size), None)
            else:
                s = lib.q2d_grad_norm(n, *args, P(1 << 20), P(1 << 21), ctypes.c_int64(size), None)
            assert s == 0, (what, s)
            got.append([(rec.recorded_launch(i).contents.name.decode(), rec.recorded_launch(i).contents.grid) for i in range(rec.recorded())])
        out.append(got)
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main(sys.argv[1])
