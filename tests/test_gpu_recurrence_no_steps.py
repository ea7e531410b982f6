"""The gated linear recurrence over sequences of no steps, by the C ABI: nothing is kept of them, and what is behind `kept` stays."""
import ctypes

import pytest
import torch

from paper_2510_05112_amd import stage_ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [1, 64, 2049])
@pytest.mark.parametrize("with_state", [False, True])
def test_nothing_is_kept_of_no_steps(width, with_state):
    lib, n = stage_ops._lib(), 3
    state = torch.randn(n, width, device="cuda") if with_state else None
    # (kept has ceil(0 / 64) = 0 blocks; the sequences of no steps need no memory either)
    guard = torch.full((4 * n * width,), 7.0, device="cuda")
    kept = guard.data_ptr() + 4 * n * width
    final = torch.full((n, width), 5.0, device="cuda")
    strides = (ctypes.c_int64 * 6)(*[width, width] * 3)
    size = lib.fpsched_op_recurrence_workspace_bytes(n, 0, width)
    assert size <= 16
    rc = lib.fpsched_op_recurrence(0, 2, n, 0, width, None, None, strides, state.data_ptr() if with_state else None, None, None, final.data_ptr(), kept, None, 0,
                                   torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    assert torch.equal(final, state if with_state else torch.zeros_like(final))
    assert bool((guard == 7).all())
    # and backward: the gradient of the state goes through, `kept` is not looked at
    grad_state, d_state = torch.randn(n, width, device="cuda"), torch.full((n, width), 5.0, device="cuda")
    strides = (ctypes.c_int64 * 10)(*[width, width] * 5)
    rc = lib.fpsched_op_recurrence_grad(0, 2, n, 0, width, None, None, None, strides, None, grad_state.data_ptr(), None, None, None, d_state.data_ptr(), None, 0,
                                        torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(d_state, grad_state)
