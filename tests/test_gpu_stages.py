"""The stage operators together: a small model's stages forward and backward against autograd in 64 bits, captured, on other streams, and measured for the tuner."""
import numpy as np
import pytest
import torch

import paper_2510_05112_amd as fp
from paper_2510_05112_amd import stages as st
from paper_2510_05112_amd import tuner
from workloads.problem import make_problem

pytestmark = pytest.mark.gpu
WIDTH, HIDDEN, VOCAB, BATCH, STEPS = 64, 96, 1000, 3, 150


def micro_batch(seed):
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(0, VOCAB, (BATCH, STEPS), generator=g)
    tokens[:, STEPS - 7 * seed - 3:] = -1
    return tokens, torch.where(tokens < 0, -1, torch.roll(tokens, -1, 1))


def in_64_bits(stages, batches, entropy_bonus):
    """Losses and the weights' gradients, by autograd from the definitions."""
    weights = [{k: w.detach().cpu().double().requires_grad_() for k, w in layer.weights.items()} for s in stages for layer in s.layers]
    layers = [layer for s in stages for layer in s.layers]
    losses = []
    for tokens, targets in batches:
        x = None
        for layer, w in zip(layers, weights):
            if isinstance(layer, st.Embedding):
                x = w["table"][tokens.clamp(min=0)] * layer.scale * (tokens >= 0)[..., None]
            elif isinstance(layer, st.Recurrence):
                gate, value = (x @ w["w"].t()).split(WIDTH, -1)
                a = torch.sigmoid(gate)
                h, hs = torch.zeros(BATCH, WIDTH, dtype=torch.float64), []
                for t in range(STEPS):
                    h = a[:, t] * h + (1 - a[:, t]) * value[:, t]
                    hs.append(h)
                x = x + torch.stack(hs, 1)
            elif isinstance(layer, st.FeedForward):
                g, u = (x @ w["w_in"].t()).split(HIDDEN, -1)
                x = x + (torch.nn.functional.silu(g) * u) @ w["w_out"].t()
            else:
                lp = torch.log_softmax(x @ w["w"].t(), -1)
                real = targets >= 0
                picked = lp.gather(-1, targets.clamp(min=0)[..., None])[..., 0]
                entropy = -(lp.exp() * lp).sum(-1)
                losses.append(-((picked + entropy_bonus * entropy) * real).sum() / real.sum())
    sum(losses).backward()
    return [float(x.detach()) for x in losses], [{k: w.grad for k, w in ws.items()} for ws in weights]


def one_f_one_b(stages, batches):
    """Two stages, two micro-batches: F0 F0 | F1 B1, F1 B1 | B0 B0, and the W items last, out of order."""
    first = [stages[0].forward(t) for t, _ in batches]
    second = [stages[1].forward(x, targets) for (x, _), (_, targets) in zip(first, batches)]
    back1 = [stages[1].input_grad(1.0, kept) for _, kept in second]
    back0 = [stages[0].input_grad(g, kept) for (g, _), (_, kept) in zip(back1, first)]
    for i in (1, 0):
        stages[0].weight_grad(first[i][1], back0[i][1])
        stages[1].weight_grad(second[i][1], back1[i][1])
    return [loss for loss, _ in second]


@pytest.fixture(scope="module")
def model():
    stages = st.language_model(2, 2, WIDTH, HIDDEN, VOCAB, dtype=torch.float16)
    stages[1].layers[-1].entropy_bonus = 0.02
    return stages


def clear(stages):
    for s in stages:
        for layer in s.layers:
            for g in layer.grads.values():
                g.zero_()


def relative(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


def test_a_models_gradients(model):
    clear(model)
    batches = [micro_batch(1), micro_batch(2)]
    losses = one_f_one_b(model, [(t.cuda(), y.cuda()) for t, y in batches])
    want, grads = in_64_bits(model, batches, 0.02)
    # Every 16-bit value on the way is off by at most 2^-11 of itself, independently of the others: a norm over thousands of them by 2^-11 / sqrt(3) for
    # each of the roundings that a result passes.  Forward a layer adds at most four in a row (product, operator, sum with x, hidden), backward as many: 24 for
    # this model of two pairs, a head and an embedding, which add up to sqrt(24) of one where they are independent, and to 24 if they were all one way.
    one = 2.0 ** -11 / 3 ** 0.5
    for got, loss in zip(losses, want):
        assert abs(float(got) - loss) <= 24 * one * abs(loss)
    for layer, grad in zip([x for s in model for x in s.layers], grads):
        for name, g in grad.items():
            assert relative(layer.grads[name], g) <= 24 * one, (type(layer).__name__, name)


def test_a_step_in_a_graph_and_eager_are_the_same(model):
    batches = [tuple(x.cuda() for x in micro_batch(i)) for i in (1, 2)]
    given = [tuple(x.clone() for x in b) for b in batches]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(2):
            clear(model)
            one_f_one_b(model, given)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for s in model:
            for layer in s.layers:
                for g in layer.grads.values():
                    g.zero_()
        losses = one_f_one_b(model, given)
    for replay in range(5):
        other = [tuple(x.cuda() for x in micro_batch((replay + i) % 7 + 1)) for i in (1, 2)]
        for to, new in zip(given, other):
            for a, b in zip(to, new):
                a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        held = [{k: g.clone() for k, g in layer.grads.items()} for s in model for layer in s.layers]
        held_losses = [x.clone() for x in losses]
        clear(model)
        eager = one_f_one_b(model, other)
        assert all(torch.equal(a, b) for a, b in zip(held_losses, eager)), replay
        for layer, grads in zip([x for s in model for x in s.layers], held):
            for name, g in grads.items():
                assert torch.equal(layer.grads[name], g), (replay, type(layer).__name__, name)


def test_operators_on_two_streams_at_once():
    ops = fp.stage_ops
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2, 2000, 64, device="cuda", generator=g).bfloat16()
    tokens = torch.randint(0, 500, (4000,), device="cuda", generator=g)
    logits = torch.randn(40, 50000, device="cuda", generator=g).half()

    def all_of_them(stream=None):
        rec = ops.gated_recurrence(x, x, keep=True, stream=stream)
        back = ops.gated_recurrence_grad(x, x, x, rec["kept"], stream=stream)
        e = ops.embedding_grad(x.view(4000, 64), tokens, 500, stream=stream)
        lp = ops.token_logprobs(logits, tokens[:40], 5, stream=stream)
        return [rec["out"], rec["state"], back["gate"], back["value"], back["state"], e, lp["logprob"], lp["entropy"], lp["ids"]]

    want = all_of_them()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [all_of_them(s) for _ in range(3) for s in streams]
    torch.cuda.synchronize()
    for found in got:
        assert all(torch.equal(a, b) for a, b in zip(found, want))


def test_workspaces_may_be_kept_and_hold_anything():
    ops = fp.stage_ops
    grad, tokens = torch.randn(3000, 40, device="cuda"), torch.randint(0, 90, (3000,), device="cuda")
    want = ops.embedding_grad(grad, tokens, 90)
    room = torch.full((32 << 20,), 0xff, dtype=torch.uint8, device="cuda")
    assert torch.equal(ops.embedding_grad(grad, tokens, 90, workspace=room), want)
    logits = torch.randn(3, 70000, device="cuda")
    want = ops.token_logprobs(logits, tokens[:3], 7)
    got = ops.token_logprobs(logits, tokens[:3], 7, workspace=room)
    x = torch.randn(1, 3000, 40, device="cuda")
    rec, again = ops.gated_recurrence(x, x), ops.gated_recurrence(x, x, workspace=room)
    assert all(torch.equal(got[k], want[k]) for k in want) and all(torch.equal(rec[k], again[k]) for k in rec)


def test_nothing_is_written_behind_the_ends():
    """Outputs with room in front and behind: the room is as it was."""
    ops = fp.stage_ops

    def between(rows, width, dtype):
        whole = torch.full(((rows + 8) * width,), 9.0, device="cuda").to(dtype)
        return whole, whole[4 * width:(rows + 4) * width].view(rows, width)

    x = torch.randn(77, 72, device="cuda").bfloat16()
    w = torch.randn(80, 72, device="cuda").bfloat16(), torch.randn(72, 40, device="cuda").bfloat16()
    logits = torch.randn(33, 5001, device="cuda")
    tokens = torch.arange(77, device="cuda")
    lp = ops.token_logprobs(logits, tokens[:33])
    for rows, width, dtype, call in ((77, 72, x.dtype, lambda out: ops.gated_ffn(x, *w, out=out)), (77, 72, x.dtype, lambda out: ops.embedding(x, tokens, out=out)),
                                     (50, 72, torch.float32, lambda out: ops.embedding_grad(x, tokens, 50, out=out)),
                                     (77, 72, x.dtype, lambda out: ops.gated_recurrence(x[None], x[None], out=out[None])),
                                     (33, 5001, torch.float32, lambda out: ops.token_logprobs_grad(logits, tokens[:33], lp["lse"], lp["entropy"], out=out))):
        whole, out = between(rows, width, dtype)
        call(out)
        assert bool((whole[:4 * width] == 9).all()) and bool((whole[(rows + 4) * width:] == 9).all())


def test_measured_costs_go_to_the_tuner():
    stages = st.language_model(4, 4, 256, 512, 32000)
    tokens = torch.randint(0, 32000, (2, 256), device="cuda")
    before = [layer.grads[k].clone() for s in stages for layer in s.layers for k in layer.grads]
    costs = tuner.measure_costs(stages, tokens, unit_us=0.5)
    after = [layer.grads[k] for s in stages for layer in s.layers for k in layer.grads]
    assert all(torch.equal(a, b) for a, b in zip(before, after))
    dur = costs["dur"]
    assert dur.shape == (8, 4) and dur.dtype == np.int32 and (dur[1:4] > 0).all() and (dur[5:7] == 0).all() and (dur[4] == dur[1]).all()
    assert (costs["kept_bytes"] > 0).all()
    whole = tuner.measure_costs(stages, tokens, split_backward=False)
    assert (whole["dur"][3] == 0).all()
    unit = int(costs["kept_bytes"].min())
    problem = make_problem(n_devices=4, n_stages=4, stage_device=[0, 1, 2, 3], n_microbatches=8, has_w=1, edges=[(0, 1, 1), (1, 2, 1), (2, 3, 1)], dur=dur,
                           mem_units=-(-costs["kept_bytes"] // unit), mem_cap=[2 ** 31 - 1] * 4)
    handle = fp.Problem(problem, tuner.stride_for(problem), device=0)
    best = tuner.tune(handle, problem, circular=False, k=3, slide=True)
    # (no schedule is shorter than its busiest device's work)
    assert best and best[0]["makespan"] >= 8 * int(dur[1:4].sum(0).max())
    handle.close()


def test_head_takes_tokens_outside_the_vocabulary_for_padding():
    head = st.Head(50, 16, torch.bfloat16)
    x = torch.randn(2, 5, 16, device="cuda").bfloat16()
    tokens = torch.randint(0, 50, (2, 5), device="cuda")
    tokens[0, 1], tokens[1, 4] = -1, -1
    other = tokens.clone()
    other[other < 0] = 50
    assert torch.equal(head.forward(x, tokens)[0], head.forward(x, other)[0])


def test_recurrence_layer_of_a_view():
    layer = st.Recurrence(16, torch.bfloat16)
    x = torch.randn(7, 3, 16, device="cuda").bfloat16()
    views, rows = x.transpose(0, 1), x.transpose(0, 1).contiguous()
    (y1, kept1), (y2, kept2) = layer.forward(views), layer.forward(rows)
    assert torch.equal(y1, y2)
    g = torch.randn_like(rows)
    assert torch.equal(layer.input_grad(g, kept1)[0], layer.input_grad(g, kept2)[0])
