"""The gradient of an embedding table for as many tokens as it takes."""
import pytest
import torch

from paper_2510_05112_amd import stage_ops as ops

pytestmark = pytest.mark.gpu


def test_gradient_of_the_most_tokens():
    # (2^26 blocks of sorted occurrences, one more than a grid has wavefronts; the last block holds all of the last row's tokens and nothing else)
    n, rows = (1 << 30) - 1, 65001
    tokens = torch.arange(n, device="cuda", dtype=torch.int32) % (rows - 1)
    tokens[[5, 1000, 1 << 20, 1 << 29, (1 << 29) + 1, n - 1]] = rows - 1
    tokens[17:26] = -1   # (of 2^30 - 1 occurrences nine are padding: 16 * (2^26 - 1) + 6)
    grad = torch.ones(n, 1, device="cuda", dtype=torch.bfloat16)
    got = ops.embedding_grad(grad, tokens, rows, out=torch.full((rows, 1), 3.0, device="cuda"))
    want = torch.bincount(tokens[tokens >= 0], minlength=rows)
    assert int(want[-1]) == 6 and int(want.max()) < 1 << 24   # (sums of ones are exact)
    assert torch.equal(got[:, 0], want.float())
    del tokens, grad, got, want
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shape", [(), (1,), (5,), (2, 3), (0, 4), (2, 3, 2)])
@pytest.mark.parametrize("width", [0, 1, 40])
def test_tokens_of_any_shape_both_ways(shape, width):
    rows = 7
    table = torch.randn(rows, width, device="cuda")
    tokens = torch.randint(0, rows, shape, device="cuda")
    got = ops.embedding(table, tokens)
    assert got.shape == (*shape, width) and torch.equal(got, table[tokens])
    grad = torch.ones_like(got)
    back = ops.embedding_grad(grad, tokens, rows)
    want = torch.bincount(tokens.reshape(-1), minlength=rows)[:, None].float().expand(rows, width)
    assert back.shape == (rows, width) and torch.equal(back, want)
    added = ops.embedding_grad(grad, tokens, rows, out=back.clone(), accumulate=True)
    assert torch.equal(added, 2 * want)
