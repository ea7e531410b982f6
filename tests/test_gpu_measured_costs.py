"""The cost table that is measured from a model's stages: what it says of memory and of time."""
import time

import numpy as np
import pytest
import torch

from paper_2510_05112_amd import stages as st
from paper_2510_05112_amd import tuner

pytestmark = pytest.mark.gpu
WIDTH, HIDDEN, VOCAB, BATCH, STEPS = 256, 512, 4096, 2, 512   # (every tensor that is kept has a multiple of 512 bytes, in which memory is handed out)
ROWS = BATCH * STEPS


def models():
    stages = st.language_model(3, 3, WIDTH, HIDDEN, VOCAB)
    return stages, torch.randint(0, VOCAB, (BATCH, STEPS), device="cuda", dtype=torch.int32)


def by_hand(split):
    """What the three stages hold of a micro-batch, in bytes."""
    x = 2 * ROWS * WIDTH
    # (x, both projections, states every 64 steps; the residual sum that the feed-forward block takes, 6 bytes for each hidden channel)
    pair = x + 2 * x + 4 * BATCH * (STEPS // 64) * WIDTH + x + 6 * ROWS * HIDDEN
    # behind B: the gradient of both projections, and the one that the block was given
    pair_b = 2 * x + x
    embedding, embedding_b = 4 * ROWS, x
    # (x, logits, whose gradient takes their place; tokens, share, log-sum-exp in two parts, entropy; the tokens are those of the first stage)
    head = x + 2 * ROWS * VOCAB + 4 * ROWS + 4 * ROWS + 8 * ROWS + 4 * ROWS
    held = [embedding + pair, pair, pair + head]
    return [h + split * b for h, b in zip(held, (embedding_b + pair_b, pair_b, pair_b))]


@pytest.mark.parametrize("split", [True, False])
def test_kept_bytes_are_what_a_stage_holds_to_its_last_backward_item(split):
    stages, tokens = models()
    costs = tuner.measure_costs(stages, tokens, split_backward=split, repeats=1)
    assert costs["kept_bytes"].tolist() == by_hand(split)


def test_kept_bytes_are_what_the_allocator_has_handed_out():
    stages, tokens = models()
    costs = tuner.measure_costs(stages, tokens, repeats=1)
    stage = stages[1]
    for _ in range(2):   # (the first: workspaces of the libraries)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        x = torch.randn(BATCH, STEPS, WIDTH, device="cuda").bfloat16()
        y, kept = stage.forward(x)
        grad = torch.ones_like(y)
        del x, y
        held_f = torch.cuda.memory_allocated() - before - grad.untyped_storage().nbytes()
        back, grad_kept = stage.input_grad(grad, kept)
        del back, grad
        held_b = torch.cuda.memory_allocated() - before
        stage.weight_grad(kept, grad_kept)
        del kept, grad_kept
    assert (held_f, held_b) == (by_hand(False)[1], by_hand(True)[1]) and costs["kept_bytes"][1] == held_b


class SlowHost(st.Layer):
    """A layer whose items take the host milliseconds and the GPU microseconds."""

    def work(self, x):
        time.sleep(0.004)
        return x + 1

    def forward(self, x):
        return self.work(x), {}

    def input_grad(self, grad, kept):
        return self.work(grad), {}

    def weight_grad(self, kept, grad_kept):
        self.done = self.work(torch.zeros(64, 64, device="cuda"))


def test_costs_are_the_gpus_and_not_what_the_host_takes_to_launch():
    stages = [st.Stage([SlowHost(), SlowHost()]) for _ in range(2)]
    costs = tuner.measure_costs(stages, torch.zeros(64, 64, device="cuda"), repeats=3)
    assert costs["us"][1:4].min() > 0 and costs["us"][1:4].max() < 1000, costs["us"]   # (8 ms of the host's)


def test_costs_of_items_that_wait_for_the_gpu_themselves():
    class Waits(SlowHost):
        def work(self, x):
            return x + float(x.sum())

    costs = tuner.measure_costs([st.Stage([Waits()])], torch.zeros(64, 64, device="cuda"), repeats=2)
    assert np.isfinite(costs["us"]).all() and (costs["dur"][1:4] > 0).all()


def test_one_micro_batch_is_held_at_a_time():
    class Large(SlowHost):
        def forward(self, x):
            return x + 1, dict(kept=torch.empty(256 << 20, dtype=torch.uint8, device="cuda"))

        def input_grad(self, grad, kept):
            return grad + 1, dict(kept=torch.empty(128 << 20, dtype=torch.uint8, device="cuda"))

    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    costs = tuner.measure_costs([st.Stage([Large()]) for _ in range(2)], torch.zeros(64, 64, device="cuda"), repeats=2)
    assert costs["kept_bytes"].tolist() == [384 << 20] * 2
    assert torch.cuda.max_memory_allocated() - before < 400 << 20


def test_items_that_wait_for_the_gpu_do_not_wait_longer_each_time():
    class Waits(SlowHost):
        times = []

        def work(self, x):
            self.times.append(time.perf_counter())
            torch.cuda.current_stream().synchronize()
            return x + 1

    tuner.measure_costs([st.Stage([Waits()])], torch.zeros(64, 64, device="cuda"), repeats=16)
    # (16 repeats behind a waiting kernel of a fraction of a millisecond; of half as much again each time, they would take half a second)
    assert Waits.times[-1] - Waits.times[6] < 0.1
