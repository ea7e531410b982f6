"""The gated feed-forward block and its gradients against the plain forms in 64 bits."""
import pytest
import torch

import paper_2510_05112_amd as fp
import stage_oracle as oracle

pytestmark = pytest.mark.gpu
ops = fp.stage_ops
TYPES = [torch.bfloat16, torch.float16]


def inputs(tokens, width, hidden, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + tokens)
    return [torch.randn(tokens, width, generator=g).to(dtype), (torch.randn(2 * hidden, width, generator=g) * width ** -0.5).to(dtype),
            (torch.randn(width, hidden, generator=g) * hidden ** -0.5).to(dtype), torch.randn(tokens, width, generator=g).to(dtype)]


def check(x, w_in, w_out, grad, act, on_gpu=None, out_dtype=None, what=""):
    dtype = x.dtype
    want = oracle.ffn(x, w_in, w_out, act, grad)
    x, w_in, w_out, grad = on_gpu or [t.cuda() for t in (x, w_in, w_out, grad)]
    done = ops.gated_ffn(x, w_in, w_out, act, keep=True)
    oracle.assert_near(done["out"], *want["out"], what + " out")
    assert torch.equal(ops.gated_ffn(x, w_in, w_out, act)["out"], done["out"])
    back = ops.gated_ffn_input_grad(grad, w_in, w_out, done["kept"], act)
    oracle.assert_near(back["x"], want["x"][0], oracle.rounded(*want["x"], dtype), what + " x")
    out = None if out_dtype is None else dict(w_in=torch.full_like(w_in, 5, dtype=out_dtype), w_out=torch.full_like(w_out, 5, dtype=out_dtype))
    weights = ops.gated_ffn_weight_grad(x, grad, done["kept"], back["kept"], out)
    for name in ("w_in", "w_out"):
        oracle.assert_near(weights[name], want[name][0], oracle.rounded(*want[name], out_dtype or dtype), what + " " + name)
    return done, back, weights


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,width,hidden", [(1, 8, 8), (2, 64, 128), (5, 256, 136), (16, 72, 264), (17, 512, 128), (33, 128, 520), (64, 192, 256), (65, 264, 40), (127, 8, 256),
                                                 (128, 128, 128), (129, 136, 392), (300, 256, 512), (513, 320, 64)])
def test_sizes(dtype, tokens, width, hidden):
    check(*inputs(tokens, width, hidden, dtype), "silu")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_activations(act):
    check(*inputs(70, 128, 192, torch.bfloat16, 1), act)
    check(*inputs(70, 128, 192, torch.float16, 1), act, out_dtype=torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
def test_enough_tiles_for_the_large_ones(dtype):
    # 2,100 x 2 x 1,304 and 2,100 x 1,288: the tiles of 256, the last ones cut off both ways; compared on some rows and columns, in 64 bits
    tokens, width, hidden = 2100, 5128, 2600
    x, w_in, w_out, grad = inputs(tokens, width, hidden, dtype, 2)
    done = ops.gated_ffn(*[t.cuda() for t in (x, w_in, w_out)], keep=True)
    back = ops.gated_ffn_input_grad(*[t.cuda() for t in (grad, w_in, w_out)], done["kept"])
    weights = ops.gated_ffn_weight_grad(x.cuda(), grad.cuda(), done["kept"], back["kept"])
    rows = torch.tensor([0, 1, 255, 256, 1023, 2047, 2048, 2099])
    want = oracle.ffn(x[rows], w_in, w_out, "silu", grad[rows])
    oracle.assert_near(done["out"].cpu()[rows], *want["out"])
    oracle.assert_near(back["x"].cpu()[rows], want["x"][0], oracle.rounded(*want["x"], dtype))
    # the weights' gradients from what was kept: products of 16-bit numbers
    for got, a, b in ((weights["w_in"], back["kept"]["pre"], x), (weights["w_out"], grad, done["kept"]["hidden"])):
        picked = torch.tensor([0, 7, 255, 256, a.shape[1] - 1])
        value, bound = oracle._product(a.cpu()[:, picked].double().t(), b.cpu().double())
        oracle.assert_near(got.cpu()[picked], value, oracle.rounded(value, bound, dtype))


def test_rows_apart():
    x, w_in, w_out, grad = inputs(40, 128, 64, torch.bfloat16, 3)
    wide = [torch.full((40, 160), float("nan")).bfloat16() for _ in range(2)]
    for w, t in zip(wide, (x, grad)):
        w[:, 16:144] = t
    on_gpu = [wide[0].cuda()[:, 16:144], w_in.cuda(), w_out.cuda(), wide[1].cuda()[:, 16:144]]
    check(x, w_in, w_out, grad, "silu", on_gpu)
    out = torch.full((40, 144), 2.0, dtype=torch.bfloat16, device="cuda")
    ops.gated_ffn(*on_gpu[:3], out=out[:, 8:136])
    assert torch.equal(out[:, 8:136], ops.gated_ffn(*on_gpu[:3])["out"]) and bool((out[:, :8] == 2).all()) and bool((out[:, 136:] == 2).all())


def test_weight_gradients_add_up_over_micro_batches():
    tokens, width, hidden = 90, 64, 72
    x, w_in, w_out, grad = inputs(tokens, width, hidden, torch.bfloat16, 4)
    want = oracle.ffn(x, w_in, w_out, "silu", grad)
    total = dict(w_in=torch.zeros(2 * hidden, width, device="cuda"), w_out=torch.zeros(width, hidden, device="cuda"))
    w = [w_in.cuda(), w_out.cuda()]
    for part in (slice(0, 33), slice(33, 33), slice(33, 90)):
        xs, gs = x[part].cuda(), grad[part].cuda()
        done = ops.gated_ffn(xs, *w, keep=True)
        back = ops.gated_ffn_input_grad(gs, *w, done["kept"])
        got = ops.gated_ffn_weight_grad(xs, gs, done["kept"], back["kept"], total, accumulate=True)
        assert got["w_in"] is total["w_in"]
    for name in total:
        oracle.assert_near(total[name], want[name][0], oracle.rounded(*want[name], torch.float32) + 2 * oracle.U * want[name][0].abs())


def test_nothing_to_do():
    x, w_in, w_out, grad = [t.cuda() for t in inputs(0, 64, 32, torch.bfloat16)]
    done = ops.gated_ffn(x, w_in, w_out, keep=True)
    back = ops.gated_ffn_input_grad(grad, w_in, w_out, done["kept"])
    out = dict(w_in=torch.full_like(w_in, 3), w_out=torch.full_like(w_out, 3))
    weights = ops.gated_ffn_weight_grad(x, grad, done["kept"], back["kept"], out)
    assert done["out"].shape == (0, 64) and not weights["w_in"].any() and not weights["w_out"].any()


def test_infinities_stay_in_their_rows():
    x, w_in, w_out, _ = inputs(140, 64, 64, torch.bfloat16, 5)
    want = ops.gated_ffn(x.cuda(), w_in.cuda(), w_out.cuda())["out"]
    x[77, 3], x[139, 0] = float("inf"), float("nan")
    got = ops.gated_ffn(x.cuda(), w_in.cuda(), w_out.cuda())["out"]
    others = torch.ones(140, dtype=torch.bool)
    others[77] = others[139] = False
    assert torch.equal(got[others.cuda()], want[others.cuda()]) and not torch.isfinite(got[139]).any()


def test_large_gates_give_finite_gradients():
    # silu and gelu are their limits there; no square overflows
    for act in ("silu", "gelu"):
        x = torch.tensor([[3e38] + [0.0] * 7, [-3e38] + [0.0] * 7, [1e20] + [0.0] * 7]).bfloat16()
        w_in, w_out = torch.zeros(16, 8).bfloat16(), torch.zeros(8, 8).bfloat16()
        w_in[0, 0], w_in[8, 0], w_out[0, 0] = 1.0, 2.0 ** -100, 1.0
        grad = torch.ones(3, 8).bfloat16()
        x, w_in, w_out, grad = [t.cuda() for t in (x, w_in, w_out, grad)]
        done = ops.gated_ffn(x, w_in, w_out, act, keep=True)
        back = ops.gated_ffn_input_grad(grad, w_in, w_out, done["kept"], act)
        # (row 0 of hidden is act(g) u = 3e38 times 3e38 / 2^100 = 2.4e8, beyond the type: infinite, and 0 times it is no number)
        assert torch.isfinite(done["out"][1:]).all() and float(done["out"][0, 0]) == float("inf"), act
        assert torch.isfinite(back["x"]).all(), act
