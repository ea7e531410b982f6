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


def form_of(dev, names, m, n):
    """Takes a product of [m][n] from the launches that are left, and says which form it has."""
    assert names.pop(0) == "gemm_kernel"
    side, places = dev.forms.pop(0)[3::4]
    (grid, block), tiles = dev.shapes.pop(0), -(-m // side) * -(-n // side)
    assert block == side * 2
    kind = "whole"
    if names and names[0] == "add_shares_kernel":
        names.pop(0)
        half = 2 if dev.forms.pop(0)[0] == 1 else 1   # (of the gated product a thread has columns of both halves)
        shared, left = divmod(dev.shapes.pop(0)[0], side * side // 8 // 256 // half)
        assert left == 0 < shared <= tiles and (grid - (tiles - shared)) % shared == 0 and grid - (tiles - shared) >= 2 * shared
        kind = "shared" if shared == tiles else "both"
    else:
        assert grid == tiles
    return f"{side} {'deep ' if places == 4 else ''}{kind}"


def ffn_forms(dev):
    from ffn_forms import FORMS
    i64, vp, size = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    end = (vp(P), size(1 << 50), None)
    seen = [set(), set(), set(), set()]
    for (t, k, f), want in FORMS.items():
        head = (0, 0, 0, i64(t), i64(k), i64(f))
        found = []
        names = dev.launched(dev.lib.fpsched_op_ffn(*head, vp(P), i64(k), vp(P), vp(P), vp(P), vp(P), vp(P), i64(k), *end))
        found += [form_of(dev, names, t, 2 * f), form_of(dev, names, t, k)]
        assert not names
        names = dev.launched(dev.lib.fpsched_op_ffn_input_grad(*head, vp(P), i64(k), vp(P), vp(P), vp(P), vp(P), i64(k), *end))
        found += [form_of(dev, names, t, f), form_of(dev, names, t, k)]
        assert not names
        for out_type, accumulate in ((0, 0), (2, 0), (2, 1)):
            names = dev.launched(dev.lib.fpsched_op_ffn_weight_grad(0, 0, *head[3:], vp(P), i64(k), vp(P), i64(k), vp(P), out_type, vp(P), vp(P), accumulate, *end))
            weights = [form_of(dev, names, 2 * f, k), form_of(dev, names, k, f)]
            assert not names and weights == list(want[4:]), ((t, k, f), weights)
        assert tuple(found + weights) == want, ((t, k, f), found + weights)
        for kinds, those in zip(seen, (want[:1], want[1:2] + want[3:4], want[2:3], want[4:])):
            kinds.update(those)
    for kinds in seen:   # (256 deep there is none)
        assert kinds >= {f"{side} {how}" for side in ("128", "256") for how in ("whole", "shared", "both")} | {"128 deep whole", "128 deep shared"}, kinds


def test_forms_of_the_feed_forward_products(stub):  # noqa: F811
    run(stub, "ffn_forms")
