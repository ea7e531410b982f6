"""The gated linear recurrence and its gradients against the plain forms in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2510_05112_amd as fp
import stage_oracle as oracle

pytestmark = pytest.mark.gpu
ops = fp.stage_ops
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def inputs(n, steps, width, dtype, seed=0):
    g = torch.Generator().manual_seed(seed + 31 * steps + width)
    gate = (2 * torch.randn(n, steps, width, generator=g) + 2).to(dtype)
    return [gate] + [torch.randn(n, steps, width, generator=g).to(dtype) for _ in range(2)] + [torch.randn(n, width, generator=g) for _ in range(2)]


def cuda(*tensors):
    return [None if t is None else t.cuda() for t in tensors]


def check(gate, value, grad, state, grad_state, lengths, on_gpu=None, what=""):
    """on_gpu: the same tensors as the operator is to have them."""
    dtype = value.dtype
    d_gate, d_value, d_grad = on_gpu if on_gpu is not None else cuda(gate, value, grad)
    d_state, d_grad_state, d_lengths = cuda(state, grad_state, lengths)
    done = ops.gated_recurrence(d_gate, d_value, d_state, d_lengths, keep=True)
    out, out_e, final, final_e, before, before_e = oracle.recurrence(gate, value, state, lengths)
    oracle.assert_near(done["out"], out, oracle.rounded(out, out_e, dtype), what + " out")
    oracle.assert_near(done["state"], final, final_e, what + " state")
    plain = ops.gated_recurrence(d_gate, d_value, d_state, d_lengths)
    assert torch.equal(plain["out"], done["out"]) and torch.equal(plain["state"], done["state"]) and "kept" not in plain
    back = ops.gated_recurrence_grad(d_grad, d_gate, d_value, done["kept"], d_grad_state, d_lengths)
    dg, dg_e, dv, dv_e, ds, ds_e = oracle.recurrence_grad(grad, gate, value, grad_state, lengths, before, before_e)
    oracle.assert_near(back["value"], dv, oracle.rounded(dv, dv_e, dtype), what + " value")
    oracle.assert_near(back["gate"], dg, oracle.rounded(dg, dg_e, dtype), what + " gate")
    oracle.assert_near(back["state"], ds, ds_e, what + " gradient of the state")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,steps,width", [(1, 1, 1), (3, 1, 130), (2, 2, 128), (1, 15, 33), (2, 16, 64), (1, 17, 129), (2, 127, 40), (2, 128, 6), (3, 129, 50), (1, 511, 2),
                                           (1, 513, 70), (2, 1100, 34), (1, 2500, 3)])
def test_sizes(dtype, n, steps, width):
    gate, value, grad, state, grad_state = inputs(n, steps, width, dtype)
    check(gate, value, grad, state, grad_state, None)
    check(gate, value, grad, None, None, None, what="without states")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("steps", [1, 40, 300, 1500])
def test_sequences_of_unequal_length(dtype, steps):
    n, width = 6, 36
    gate, value, grad, state, grad_state = inputs(n, steps, width, dtype, 1)
    lengths = torch.tensor([0, 1, steps, steps + 9, -3, (2 * steps + 2) // 3], dtype=torch.int32)
    check(gate, value, grad, state, grad_state, lengths)
    # what is behind a sequence's end is not looked at
    behind = torch.arange(steps)[None] >= lengths[:, None]
    nan = [torch.where(behind[..., None], float("nan"), t.float()).to(dtype).cuda() for t in (gate, value, grad)]
    check(gate, value, grad, state, grad_state, lengths, nan, "with NaN behind the ends")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(dtype):
    n, steps, width = 3, 200, 66
    gate, value, grad, state, grad_state = inputs(n, steps, width, dtype, 2)
    by_step = [t.cuda().transpose(0, 1).contiguous().transpose(0, 1) for t in (gate, value, grad)]
    check(gate, value, grad, state, grad_state, None, by_step, "steps outermost")
    for first in (0, 1, 2):
        wide = [torch.full((n, steps, width + 6), 9.0).to(dtype) for _ in range(3)]
        for w, t in zip(wide, (gate, value, grad)):
            w[..., first:first + width] = t
        check(gate, value, grad, state, grad_state, None, [w.cuda()[..., first:first + width] for w in wide], f"channels from {first}")
    shared = gate[:1].expand(n, steps, width)
    check(shared, value, grad, state, grad_state, None, [gate[:1].cuda().expand(n, steps, width), value.cuda(), grad.cuda()], "one gate for all sequences")


def test_output_is_written_where_it_is_wanted():
    gate, value, _, state, _ = cuda(*inputs(2, 70, 20, torch.float32, 3))
    want = ops.gated_recurrence(gate, value, state)
    out = torch.full((70, 2, 24), 4.0, device="cuda")
    got = ops.gated_recurrence(gate, value, state, out=out[..., 2:22].transpose(0, 1), final_state=state)
    assert torch.equal(got["out"], want["out"]) and got["state"] is state and torch.equal(state, want["state"])
    assert bool((out[..., :2] == 4).all()) and bool((out[..., 22:] == 4).all())


@pytest.mark.parametrize("steps,width", [(40, 64), (4000, 66)])
def test_the_state_may_be_updated_in_place(steps, width):
    # (4000 steps of 66 channels are cut into segments, whose workgroups begin at different times)
    gate, value, grad, state, grad_state = cuda(*inputs(2, steps, width, torch.bfloat16, 4))
    want = ops.gated_recurrence(gate, value, state, keep=True)
    held = state.clone()
    got = ops.gated_recurrence(gate, value, held, final_state=held)
    assert torch.equal(held, want["state"]) and torch.equal(got["out"], want["out"])


def test_step_by_step_is_the_whole():
    n, steps, width = 5, 30, 48
    gate, value, _, state, _ = inputs(n, steps, width, torch.float32, 5)
    out, out_e, final, final_e, _, _ = oracle.recurrence(gate, value, state, None)
    gate, value, held = cuda(gate, value, state)
    for t in range(steps):
        done = ops.gated_recurrence(gate[:, t:t + 1], value[:, t:t + 1], held, final_state=held)
        oracle.assert_near(done["out"][:, 0], out[:, t], oracle.rounded(out[:, t], out_e[:, t], torch.float32), f"step {t}")
    oracle.assert_near(held, final, final_e)


def test_a_sequence_in_pieces_is_the_whole_and_so_are_its_gradients():
    n, steps, width, at = 2, 700, 40, 333
    gate, value, grad, state, grad_state = inputs(n, steps, width, torch.float32, 6)
    _, _, _, _, before, before_e = oracle.recurrence(gate, value, state, None)
    dg, dg_e, dv, dv_e, ds, ds_e = oracle.recurrence_grad(grad, gate, value, grad_state, None, before, before_e)
    gate, value, grad, state, grad_state = cuda(gate, value, grad, state, grad_state)
    one = ops.gated_recurrence(gate[:, :at], value[:, :at], state, keep=True)
    two = ops.gated_recurrence(gate[:, at:], value[:, at:], one["state"], keep=True)
    back2 = ops.gated_recurrence_grad(grad[:, at:], gate[:, at:], value[:, at:], two["kept"], grad_state)
    back1 = ops.gated_recurrence_grad(grad[:, :at], gate[:, :at], value[:, :at], one["kept"], back2["state"])
    oracle.assert_near(torch.cat([back1["gate"], back2["gate"]], 1), dg, oracle.rounded(dg, dg_e, torch.float32))
    oracle.assert_near(torch.cat([back1["value"], back2["value"]], 1), dv, oracle.rounded(dv, dv_e, torch.float32))
    oracle.assert_near(back1["state"], ds, ds_e)


def test_gates_at_their_limits():
    # gates that keep everything, nothing, or are no number: in their own channel only
    gate = torch.zeros(1, 50, 6)
    gate[..., 0], gate[..., 1], gate[..., 2], gate[..., 3], gate[..., 4] = float("inf"), float("-inf"), 88.0, -88.0, float("nan")
    value, state = torch.randn(1, 50, 6), torch.randn(1, 6)
    got = ops.gated_recurrence(gate.cuda(), value.cuda(), state.cuda())["out"].cpu()
    assert torch.equal(got[..., 0], state[:, None, 0].expand(1, 50)) and torch.equal(got[..., 1], value[..., 1])
    assert torch.isnan(got[..., 4]).all() and not torch.isnan(got[..., [0, 1, 2, 3, 5]]).any()
    out, out_e, *_ = oracle.recurrence(gate, value, state, None)
    oracle.assert_near(got[..., 2:4], out[..., 2:4], oracle.rounded(out, out_e, torch.float32)[..., 2:4])


def test_gradients_against_differences():
    n, steps, width = 1, 9, 4
    gate, value, grad, state, grad_state = inputs(n, steps, width, torch.float32, 7)

    def total(gate, value, state):
        out, _, final, *_ = oracle.recurrence(gate, value, state, None)
        return float((out * grad.double()).sum() + (final * grad_state.double()).sum())

    done = ops.gated_recurrence(gate.cuda(), value.cuda(), state.cuda(), keep=True)
    back = ops.gated_recurrence_grad(grad.cuda(), gate.cuda(), value.cuda(), done["kept"], grad_state.cuda())
    step = 1e-4
    whole = [gate.double(), value.double(), state.double()]
    for which, name in enumerate(("gate", "value", "state")):
        got = back[name].cpu().reshape(-1)
        for i in range(0, got.numel(), 5):
            up, down = [t.clone() for t in whole], [t.clone() for t in whole]
            up[which].reshape(-1)[i] += step
            down[which].reshape(-1)[i] -= step
            want = (total(*up) - total(*down)) / (2 * step)
            # the difference's own error: step^2 / 6 times a third derivative (of sums of at most nine terms of size a few: under 100), and 64-bit rounding / step
            assert abs(float(got[i]) - want) <= 2e-6 + 1e-5 * abs(want), (name, i)


def test_nothing_to_do():
    state = torch.randn(3, 10, device="cuda")
    none = torch.empty(3, 0, 10, device="cuda")
    done = ops.gated_recurrence(none, none, state, keep=True)
    assert done["out"].shape == (3, 0, 10) and torch.equal(done["state"], state)
    back = ops.gated_recurrence_grad(none, none, none, done["kept"], state)
    assert torch.equal(back["state"], state) and back["gate"].shape == (3, 0, 10)
    empty = torch.empty(0, 5, 10, device="cuda")
    assert ops.gated_recurrence(empty, empty)["out"].shape == (0, 5, 10)


def test_offsets_beyond_32_bits():
    # the last of 70,000 steps that are 65,536 elements apart
    steps, width = 70000, 4
    store = torch.zeros(steps, 65536, dtype=torch.float16, device="cuda")
    gate, value, grad, _, _ = inputs(1, steps, width, torch.float16, 8)
    store[:, 8:8 + width] = value[0].cuda()
    got = ops.gated_recurrence(gate.cuda(), store[None, :, 8:8 + width], keep=True)
    want = ops.gated_recurrence(gate.cuda(), value.cuda(), keep=True)
    assert torch.equal(got["out"], want["out"])
    back = [ops.gated_recurrence_grad(grad.cuda(), gate.cuda(), v, want["kept"]) for v in (store[None, :, 8:8 + width], value.cuda())]
    assert all(torch.equal(back[0][k], back[1][k]) for k in back[0])


@pytest.mark.parametrize("width", [1, 6, 130])
def test_many_segments(width):
    # (one long sequence of few channels: a thousand segments, whose maps are composed by shares)
    steps = 70001
    g = torch.Generator().manual_seed(width)
    gate, value, grad = (torch.randn(1, steps, width, generator=g) for _ in range(3))
    a, v, d = torch.sigmoid(gate.double())[0].numpy(), value.double()[0].numpy(), grad.double()[0].numpy()
    out, behind = np.empty_like(v), np.empty_like(v)
    h = e = np.zeros(width)
    for t in range(steps):
        h = out[t] = a[t] * h + (1 - a[t]) * v[t]
    for t in range(steps - 1, -1, -1):
        behind[t] = d[t] + e
        e = a[t] * behind[t]
    done = ops.gated_recurrence(gate.cuda(), value.cuda(), keep=True)
    # (a state forgets: a mean of values of 5 at most, its terms off by some 2^-21 of themselves; the gradient likewise)
    assert np.abs(done["out"][0].cpu().double().numpy() - out).max() <= 1e-5
    back = ops.gated_recurrence_grad(grad.cuda(), gate.cuda(), value.cuda(), done["kept"])
    assert np.abs(back["value"][0].cpu().double().numpy() - behind * (1 - a)).max() <= 1e-5 * (1 + np.abs(behind).max())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,steps,width", [(5, 7, 33), (5, 8, 34), (5, 9, 34), (300, 9, 34), (300, 16, 130), (260, 16, 33), (300, 17, 34), (3, 16, 200)])
def test_few_steps(dtype, n, steps, width):
    gate, value, grad, state, grad_state = inputs(n, steps, width, dtype, 7)
    check(gate, value, grad, state, grad_state, None)
    lengths = torch.randint(0, steps + 1, (n,), generator=torch.Generator().manual_seed(steps), dtype=torch.int32)
    lengths[0], lengths[1] = 0, steps
    check(gate, value, grad, state, None, lengths)
