"""The feed-forward block's items on two streams at once, with workspaces of the caller's, and captured, where tiles are shared over k."""
import pytest
import torch

from paper_2510_05112_amd import stage_ops as ops
from test_gpu_ffn import inputs

pytestmark = pytest.mark.gpu
SIZES = [(5, 520, 264), (40, 1288, 4104), (1040, 64, 776)]   # few rows; shares of k in every product of the second, in three of the third


def items(x, w_in, w_out, grad, stream=None, workspace=None):
    done = ops.gated_ffn(x, w_in, w_out, keep=True, stream=stream, workspace=workspace)
    back = ops.gated_ffn_input_grad(grad, w_in, w_out, done["kept"], stream=stream, workspace=workspace)
    weights = ops.gated_ffn_weight_grad(x, grad, done["kept"], back["kept"], stream=stream, workspace=workspace)
    return [done["out"], back["x"], weights["w_in"], weights["w_out"]]


@pytest.mark.parametrize("sizes", SIZES)
def test_two_streams_at_once(sizes):
    on = [t.cuda() for t in inputs(*sizes, torch.bfloat16, 1)]
    want = items(*on)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [items(*on, stream=s) for _ in range(4) for s in streams]
    torch.cuda.synchronize()
    for found in got:
        assert all(torch.equal(a, b) for a, b in zip(found, want))


@pytest.mark.parametrize("sizes", SIZES)
def test_workspaces_may_be_kept_and_hold_anything(sizes):
    on = [t.cuda() for t in inputs(*sizes, torch.float16, 2)]
    want = items(*on)
    size = ops._lib().fpsched_op_ffn_workspace_bytes(*sizes)
    room = torch.full((size + 512,), 0xff, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        assert all(torch.equal(a, b) for a, b in zip(items(*on, workspace=room[:size]), want))
        assert bool((room[size:] == 0xff).all())
        room[:size] = 0x7f


@pytest.mark.parametrize("sizes", SIZES)
def test_captured_and_replayed(sizes):
    on = [t.cuda() for t in inputs(*sizes, torch.bfloat16, 3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        items(*on)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):   # (two graphs over the same inputs, each with memory of its own)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            found = items(*on)
        graphs.append((graph, found))
    for replay in range(4):
        for to, new in zip(on, inputs(*sizes, torch.bfloat16, 10 + replay)):
            to.copy_(new)
        want = items(*on)
        for graph, found in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(found, want)), replay
