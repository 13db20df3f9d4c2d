"""Grids of matrices whose tiles pass what one dimension of a launch takes (work-items below 2^32), on a
stand-in for the HIP runtime that refuses launches as it does and runs nothing."""
import ctypes
import json
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
LIB = os.path.join(os.path.dirname(HERE), "paper_2607_24953_amd", "libq2d.so")
FMTS = {"fp4": 0, "mxfp8": 1, "fp4_1d": 2}
# rows, columns: tiles of 128 x 256 up to the 2^23 that fill one dimension with 512 lanes each, and beyond
SIZES = [(2 ** 30 - 128, 1), (2 ** 30, 1), (2 ** 30 + 129, 128), (2 ** 31 - 1, 1), (128, 2 ** 27), (2 ** 17, 2 ** 21 + 300)]

RECORDER = """
#define hipLaunchKernel recorded_launch_kernel
#include "launch_recorder.c"
#undef hipLaunchKernel
static uint64_t last[3];
int hipLaunchKernel(const void *fn, dim3 grid, dim3 block, void **args, size_t lds, void *stream)
{
    last[0] = grid.x; last[1] = grid.y; last[2] = grid.z;
    if ((uint64_t)grid.x * block.x >= 1ull << 32 || grid.y > 65535 || grid.z > 65535) return 1;
    return recorded_launch_kernel(fn, grid, block, args, lds, stream);
}
const uint64_t *last_grid(void) { return last; }
"""


class _Norm(ctypes.Structure):
    """q2d_rmsnorm."""
    _fields_ = [("x_dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32),
                ("y_dtype", ctypes.c_int32), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("eps", ctypes.c_double),
                ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("residual", ctypes.c_void_p), ("ld_residual", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("h", ctypes.c_void_p), ("ldh", ctypes.c_int64), ("y", ctypes.c_void_p),
                ("ldy", ctypes.c_int64), ("rstd", ctypes.c_void_p)]


def run(tmp_path, calls):
    if shutil.which("gcc") is None:
        pytest.skip("gcc not found")
    src, so = os.path.join(str(tmp_path), "recorder.c"), os.path.join(str(tmp_path), "recorder.so")
    with open(src, "w") as f:
        f.write(RECORDER)
    subprocess.run(["gcc", "-std=c99", "-O1", "-Wall", "-shared", "-fPIC", "-I", HERE, "-o", so, src], check=True)
    p = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(calls), capture_output=True, text=True,
                       timeout=300)
    assert p.returncode == 0, p.stderr[-4000:]
    return json.loads(p.stdout)


def tiles(rows, cols):
    return -(-rows // 128) * -(-cols // 256)


def test_dequantize(tmp_path):
    calls = [dict(fn="dequantize", fmt=f, rows=r, cols=c, copy=k, dt=d) for f in FMTS for r, c in SIZES for k in (0, 1) for d in (0, 1)]
    for c, (status, launch, grid) in zip(calls, run(tmp_path, calls)):
        assert status == 0 and "dequantize_kernel" in launch[0] and launch[1] == 512, (c, status)
        n = grid[0] * grid[1] * grid[2]
        assert tiles(c["rows"], c["cols"]) <= n < tiles(c["rows"], c["cols"]) + 2 ** 20, (c, grid)
    # more than any launch takes
    for r, c in ((2 ** 31, 2 ** 31), (2 ** 31, 2 ** 20 * 9)):
        assert [x[0] for x in run(tmp_path, [dict(fn="dequantize", fmt="fp4", rows=r, cols=c, copy=0, dt=0)])] == [2]


def test_norm_operands(tmp_path):
    sizes = [x for x in SIZES if x[1] <= 2 ** 27]
    calls = [dict(fn="norm", fmt=f, rows=r, cols=c, dt=d) for f in (["fp4"], ["mxfp8"], ["fp4_1d"], ["fp4", "mxfp8"]) for r, c in sizes
             for d in (0, 1)]
    for c, (status, launch, grid) in zip(calls, run(tmp_path, calls)):
        assert status == 0 and "rmsnorm_quantize_kernel" in launch[0] and launch[1] == 512, (c, status)
        n = grid[0] * grid[1] * grid[2]
        assert tiles(c["rows"], c["cols"]) <= n < tiles(c["rows"], c["cols"]) + 2 ** 20, (c, grid)
    # more than any launch takes
    assert [x[0] for x in run(tmp_path, [dict(fn="norm", fmt=["fp4"], rows=2 ** 31 - 1, cols=2 ** 21, dt=1)])] == [2]


def _main(so):
    class Launch(ctypes.Structure):
        _fields_ = [("name", ctypes.c_char_p), ("grid", ctypes.c_uint32), ("block", ctypes.c_uint32), ("lds", ctypes.c_uint64)]
    rec = ctypes.CDLL(so, mode=ctypes.RTLD_GLOBAL)
    rec.recorded_launch.restype = ctypes.POINTER(Launch)
    rec.last_grid.restype = ctypes.POINTER(ctypes.c_uint64)
    sys.path.insert(0, HERE)
    from launches import _Tensor
    lib = ctypes.CDLL(LIB)
    P, I64 = ctypes.c_void_p, ctypes.c_int64
    place = 1 << 50                                     # apart, whatever the size

    def tensor(fmt, rows, cols, at):
        t = _Tensor()
        assert lib.q2d_tensor_init(ctypes.byref(t), FMTS[fmt], I64(rows), I64(cols), 32, None) == 0
        t.codes, t.codes_t, t.scales, t.scales_t = (place * (at + i) for i in range(4))
        return t

    out = []
    for c in json.load(sys.stdin):
        rec.record_clear()
        if c["fn"] == "dequantize":
            t = tensor(c["fmt"], c["rows"], c["cols"], 2)
            s = lib.q2d_dequantize(ctypes.byref(t), c["copy"], P(place), c["dt"], I64(c["cols"]), None, I64(0), None)
        else:
            n = _Norm(x_dtype=c["dt"], rows=c["rows"], cols=c["cols"], eps=1e-5, x=place, ldx=c["cols"], weight=2 * place, rstd=3 * place)
            q = {f == "mxfp8": tensor(f, c["rows"], c["cols"], 4 + 4 * i) for i, f in enumerate(c["fmt"])}
            s = lib.q2d_rmsnorm_fwd(ctypes.byref(n), *(ctypes.byref(q[k]) if k in q else None for k in (False, True)), None)
        n = rec.recorded()
        l = rec.recorded_launch(n - 1).contents if n else None
        out.append((s, (l.name.decode(), l.block) if n else None, rec.last_grid()[:3]))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main(sys.argv[1])
