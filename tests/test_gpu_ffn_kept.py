"""What a feed-forward block keeps serves one B item, and then its W items; calls in another order are refused."""
import copy

import pytest
import torch

from paper_2510_05112_amd import stage_ops as ops
from paper_2510_05112_amd import stages as st

pytestmark = pytest.mark.gpu


def block(tokens=40, width=64, hidden=72):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, w_in, w_out, grad = (torch.randn(*shape, device="cuda", generator=g).bfloat16() for shape in ((tokens, width), (2 * hidden, width), (width, hidden), (tokens, width)))
    return x, w_in, w_out, grad


@pytest.mark.parametrize("tokens", [0, 1, 40])
def test_items_out_of_order(tokens):
    x, w_in, w_out, grad = block(tokens)
    kept = ops.gated_ffn(x, w_in, w_out, keep=True)["kept"]
    for held in (kept, dict(kept), dict(x=x, **kept), copy.copy(kept)):   # (the layers put it beside their own)
        with pytest.raises(ValueError, match="gated_ffn_input_grad"):
            ops.gated_ffn_weight_grad(x, grad, kept, held)                   # W before B
    again = dict(kept)
    back = ops.gated_ffn_input_grad(grad, w_in, w_out, kept)
    for held in (kept, again, back["kept"], dict(back["kept"])):
        with pytest.raises(ValueError, match="once"):
            ops.gated_ffn_input_grad(grad, w_in, w_out, held)                # B again
    # W as often as wanted, with the same bits
    one, two = (ops.gated_ffn_weight_grad(x, grad, kept, back["kept"]) for _ in range(2))
    assert all(torch.equal(one[k], two[k]) for k in one)
    # an R item keeps anew
    fresh = ops.gated_ffn(x, w_in, w_out, keep=True)["kept"]
    second = ops.gated_ffn_input_grad(grad, w_in, w_out, fresh)
    assert torch.equal(second["x"], back["x"])


def test_a_call_that_was_refused_has_taken_nothing():
    x, w_in, w_out, grad = block()
    want = ops.gated_ffn_input_grad(grad, w_in, w_out, ops.gated_ffn(x, w_in, w_out, keep=True)["kept"])["x"]
    kept = ops.gated_ffn(x, w_in, w_out, keep=True)["kept"]
    for wrong in (lambda: ops.gated_ffn_input_grad(grad[:, :56], w_in, w_out, kept), lambda: ops.gated_ffn_input_grad(grad, w_in, w_out, kept, "tanh"),
                  lambda: ops.gated_ffn_input_grad(grad, w_in, w_out, kept, workspace=torch.zeros(4, device="cuda", dtype=torch.uint8)[1:2].cpu())):
        with pytest.raises(ValueError):
            wrong()
    assert torch.equal(ops.gated_ffn_input_grad(grad, w_in, w_out, kept)["x"], want)


def test_layers_out_of_order():
    layer = st.FeedForward(64, 72, torch.bfloat16)
    x = torch.randn(2, 20, 64, device="cuda").bfloat16()
    y, kept = layer.forward(x)
    grad = torch.ones_like(y)
    _, grad_kept = layer.input_grad(grad, kept)
    with pytest.raises(ValueError, match="once"):
        layer.input_grad(grad, kept)
    layer.weight_grad(kept, grad_kept)
    assert st.kept_bytes(kept) == 2 * x.numel() + 6 * 40 * 72   # (x, and g and u in 24 bits)


def test_what_is_kept_is_tensors_alone():
    x, w_in, w_out, grad = block()
    kept = ops.gated_ffn(x, w_in, w_out, keep=True)["kept"]
    back = ops.gated_ffn_input_grad(grad, w_in, w_out, kept)["kept"]
    for held in (kept, back):
        assert set(held) == {"pre", "hidden"} and all(torch.is_tensor(t) for t in held.values())
