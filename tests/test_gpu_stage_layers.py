"""The layers of a model's stages: their weights' gradients in 32 bits, micro-batches of any size and inputs that are views."""
import pytest
import torch

import stage_oracle as oracle
from paper_2510_05112_amd import stages as st
from paper_2510_05112_amd import tuner

pytestmark = pytest.mark.gpu


def items(layer, a, b):
    """The W item of a layer whose weights' gradient is a^T b."""
    if isinstance(layer, st.Head):
        layer.weight_grad(dict(x=b), dict(logits=a))
    else:
        layer.weight_grad(dict(x=b), dict(both=a))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["recurrence", "head"])
def test_weight_gradients_add_up_in_32_bits(kind, dtype):
    width, vocab, rows, batches = 64, 200, 130, 12
    layer = st.Recurrence(width, dtype) if kind == "recurrence" else st.Head(vocab, width, dtype)
    g = torch.Generator().manual_seed(3)
    total, bound = torch.zeros(layer.grads["w"].shape, dtype=torch.float64), 0.0
    for _ in range(batches):
        a, b = (torch.randn(rows, n, generator=g).to(dtype) for n in layer.weights["w"].shape)
        items(layer, a.cuda(), b.cuda())
        product, off = oracle._product(a.double().t(), b.double())
        if dtype == torch.float32:   # (of 32-bit factors a product is rounded too)
            off = 2 * off
        total = total + product
        # (adding to the sum rounds it once more)
        bound = bound + off + oracle.U * (total.abs() + off)
    oracle.assert_near(layer.grads["w"], total, bound, kind)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("kind", ["recurrence", "head"])
def test_weight_gradients_of_whole_numbers_are_exact(kind, dtype):
    # (130 products of 0 to 225: sums of up to 15 bits a micro-batch and of 19 in all, which 32 bits hold and 16 do not)
    width, vocab, rows, batches = 64, 200, 130, 12
    layer = st.Recurrence(width, dtype) if kind == "recurrence" else st.Head(vocab, width, dtype)
    g = torch.Generator().manual_seed(5)
    total = torch.zeros(layer.grads["w"].shape, dtype=torch.float64)
    for _ in range(batches):
        a, b = (torch.randint(0, 16, (rows, n), generator=g).to(dtype) for n in layer.weights["w"].shape)
        items(layer, a.cuda(), b.cuda())
        total += a.double().t() @ b.double()
    assert torch.equal(layer.grads["w"].double().cpu(), total)


@pytest.mark.parametrize("kind", ["recurrence", "head"])
def test_weight_gradients_beyond_float16(kind):
    layer = st.Recurrence(16, torch.float16) if kind == "recurrence" else st.Head(32, 16, torch.float16)
    n = layer.weights["w"].shape[0]
    items(layer, torch.full((8, n), 300.0, device="cuda").half(), torch.full((8, 16), 300.0, device="cuda").half())
    assert bool((layer.grads["w"] == 8 * 300.0 * 300.0).all())
    layer.grads["w"].zero_()
    items(layer, torch.full((1, n), 2.0 ** -14, device="cuda").half(), torch.full((1, 16), 2.0 ** -14, device="cuda").half())
    assert bool((layer.grads["w"] == 2.0 ** -28).all())


@pytest.mark.parametrize("batch,steps", [(0, 5), (3, 0), (0, 0)])
def test_a_micro_batch_of_no_tokens(batch, steps):
    """(A shard of a batch that has none.)  Nothing is added to the gradients."""
    model = st.language_model(2, 2, 64, 96, 500)
    tokens = torch.zeros(batch, steps, dtype=torch.int64, device="cuda")
    x, kept0 = model[0].forward(tokens)
    loss, kept1 = model[1].forward(x, tokens)
    assert x.shape == (batch, steps, 64) and float(loss) == 0
    grad, grad_kept1 = model[1].input_grad(1.0, kept1)
    assert grad.shape == x.shape
    none, grad_kept0 = model[0].input_grad(grad, kept0)
    assert none is None
    for stage, kept, grad_kept in zip(model, (kept0, kept1), (grad_kept0, grad_kept1)):
        stage.weight_grad(kept, grad_kept)
        assert not any(bool(g.any()) for layer in stage.layers for g in layer.grads.values())


def test_tokens_that_are_views():
    # (a text's tokens but the last, and those behind each)
    model = st.language_model(2, 2, 64, 96, 500)
    text = torch.randint(0, 500, (3, 41), device="cuda")
    tokens, targets = text[:, :-1], text[:, 1:]
    for of, to in ((tokens, targets), (tokens.t(), targets.t())):
        x, kept0 = model[0].forward(of)
        want, _ = model[0].forward(of.contiguous())
        assert torch.equal(x, want)
        loss, kept1 = model[1].forward(x, to)
        assert torch.equal(loss, model[1].forward(want, to.contiguous())[0])
        grad, _ = model[1].input_grad(1.0, kept1)
        _, grad_kept0 = model[0].input_grad(grad, kept0)
        model[0].weight_grad(kept0, grad_kept0)
    costs = tuner.measure_costs(model, tokens, targets, repeats=1)
    assert (costs["dur"][1:4] > 0).all()
