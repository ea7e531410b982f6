"""Every form of the feed-forward block's products against the plain forms in 64 bits: rows, and columns of the weights' gradients, out of every tile."""
import pytest
import torch

import stage_oracle as oracle
from ffn_forms import FORMS
from paper_2510_05112_amd import stage_ops as ops
from test_gpu_ffn import inputs

pytestmark = pytest.mark.gpu


def some(n, apart):
    """Some of n, in every tile of 128, with the ends of the tiles and the last ones."""
    edges = [i + d for i in range(0, n + 128, 128) for d in (-1, 0)]
    return torch.tensor(sorted({i for i in list(range(3, n, apart)) + edges + [n - 1] if 0 <= i < n}))


@pytest.mark.parametrize("sizes", FORMS)
def test_forms(sizes):
    tokens, width, hidden = sizes
    number = list(FORMS).index(sizes)
    dtype, act = (torch.bfloat16, torch.float16)[number % 2], ("silu", "gelu", "relu")[number % 3]
    x, w_in, w_out, grad = inputs(tokens, width, hidden, dtype, number)
    on = [t.cuda() for t in (x, w_in, w_out, grad)]
    done = ops.gated_ffn(*on[:3], act, keep=True)
    assert torch.equal(ops.gated_ffn(*on[:3], act)["out"], done["out"])
    back = ops.gated_ffn_input_grad(on[3], *on[1:3], done["kept"], act)
    rows = some(tokens, 97)
    want = oracle.ffn(x[rows], w_in, w_out, act, grad[rows])
    oracle.assert_near(done["out"][rows.cuda()], *want["out"], "out")
    oracle.assert_near(back["x"][rows.cuda()], want["x"][0], oracle.rounded(*want["x"], dtype), "x")
    # The weights' gradients are products of what B left, whose rows are as good as the two results that were made of them.
    g = torch.Generator().manual_seed(number)
    pairs = dict(w_in=(back["kept"]["pre"].cpu(), x), w_out=(grad, back["kept"]["hidden"].cpu()))
    old = {name: torch.randn(a.shape[1], b.shape[1], generator=g) for name, (a, b) in pairs.items()}
    sixteen = ops.gated_ffn_weight_grad(on[0], on[3], done["kept"], back["kept"])
    plain = ops.gated_ffn_weight_grad(on[0], on[3], done["kept"], back["kept"], {name: torch.full_like(t, 5, device="cuda") for name, t in old.items()})
    added = ops.gated_ffn_weight_grad(on[0], on[3], done["kept"], back["kept"], {name: t.cuda() for name, t in old.items()}, accumulate=True)
    for name, (a, b) in pairs.items():
        picked = some(a.shape[1], 211)
        value, bound = oracle._product(a[:, picked].double().t(), b.double())
        before = old[name][picked].double()
        for got, expected, off, kind in ((sixteen, value, bound, dtype), (plain, value, bound, torch.float32), (added, value + before, bound, torch.float32)):
            oracle.assert_near(got[name][picked.cuda()], expected, oracle.rounded(expected, off, kind), name)
