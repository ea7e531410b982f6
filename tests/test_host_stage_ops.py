"""Which kernels the stage operators launch, without a GPU, and with which grids: every test runs in a process of its own in which a stand-in for the
HIP runtime comes before the real one (see test_host_launches)."""
import ctypes
import os
import pickle
import subprocess
import sys

from test_host_launches import HERE, pytestmark, stub  # noqa: F401

P = 1 << 20   # a pointer that nothing looks at
LANES = (1 << 32) - 1   # of a grid's x


def run(stub, what, *args):  # noqa: F811
    """Runs the function `what` of this file in a new process, with the stand-in."""
    code = (f"import pickle, sys; sys.path[:0] = [{HERE!r}, {os.path.dirname(HERE)!r}]; import test_host_launches as t, test_host_stage_ops as o; "
            f"o.{what}(t.Device({stub!r}), *pickle.loads(sys.stdin.buffer.read()))")
    done = subprocess.run([sys.executable, "-c", code], input=pickle.dumps(args), stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    assert done.returncode == 0, done.stdout.decode()


def embedding_grad(dev, n, rows, width=1, type_=2):
    f = dev.lib.fpsched_op_embedding_grad
    i64, vp = ctypes.c_int64, ctypes.c_void_p
    rc = f(0, type_, vp(P), i64(width), i64(rows), i64(width), vp(P), 0, i64(n), ctypes.c_float(1), type_, vp(P), i64(width), 0, vp(P), ctypes.c_size_t(1 << 50), None)
    return dev.launched(rc)


def most_tokens(dev):
    for n in ((1 << 30) - 1, (1 << 30) - 16, (1 << 30) - 17, 1000):
        names = embedding_grad(dev, n, 70000)
        assert all(0 < grid * block <= LANES for grid, block in dev.shapes), (n, dev.shapes)
        sums = [grid for name, (grid, _) in zip(names, dev.shapes) if name == "row_sums_kernel"]
        assert sum(sums) == -(-n // 16), (n, sums)
    # the largest table: four passes of the sort
    assert embedding_grad(dev, 20000, (1 << 31) - 1).count("sort_place_kernel") == 4


def test_most_tokens_and_rows_of_a_tables_gradient(stub):  # noqa: F811
    run(stub, "most_tokens")
