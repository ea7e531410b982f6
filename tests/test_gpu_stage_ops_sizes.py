"""The largest sizes that the stage operators take in one dimension: ids, steps and places beyond 31 bits of bytes."""
import math

import pytest
import torch

from paper_2510_05112_amd import stage_ops as ops

pytestmark = pytest.mark.gpu
MOST = (1 << 31) - 1


@pytest.fixture(autouse=True)
def memory_is_given_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("k", [0, 4])
def test_log_probabilities_over_the_largest_vocabulary(k):
    logits = torch.zeros(1, MOST, dtype=torch.bfloat16, device="cuda")
    at, peaks = [MOST - 1, 5, 1 << 30], [20.0, 19.0, 18.0]
    for i, x in zip(at, peaks):
        logits[0, i] = x
    tokens = torch.tensor([MOST - 1], device="cuda")
    total = sum(math.exp(x) for x in peaks) + MOST - 3
    done = ops.token_logprobs(logits, tokens, k)
    # (a lane adds 8,192 ones and less, exactly; its sum, exp and log by a few roundings each)
    assert abs(float(done["logprob"]) - (20 - math.log(total))) < 1e-5
    want_h = math.log(total) - sum(x * math.exp(x) for x in peaks) / total
    assert abs(float(done["entropy"]) - want_h) < 1e-4
    if k:
        assert done["ids"][0].tolist() == [*at, 0]
        assert all(abs(float(a) - (x - math.log(total))) < 1e-5 for a, x in zip(done["logprobs"][0], [*peaks, 0.0]))
    ops.token_logprobs_grad(logits, tokens, done["lse"], done["entropy"], torch.full((1,), 3.0, device="cuda"), out=logits)
    for i, x in zip([*at, 0, MOST - 2], [*peaks, 0.0, 0.0]):
        p = math.exp(x) / total
        want = 3 * ((i == MOST - 1) - p)
        assert abs(float(logits[0, i]) - want) <= 2.0 ** -8 * abs(want) + 1e-4 * 3 * p, i


def test_recurrence_of_the_most_steps():
    # (gates that let nothing through: a step is its value, and its gradient is that of its value)
    value = (torch.arange(MOST, device="cuda", dtype=torch.int32) % 251).bfloat16()[None, :, None]
    gate = torch.full_like(value, -math.inf)
    done = ops.gated_recurrence(gate, value, torch.ones(1, 1, device="cuda"), keep=True)
    assert torch.equal(done["out"], value) and float(done["state"]) == (MOST - 1) % 251
    assert torch.equal(done["kept"][0, 1:, 0], value[0, 63:-1:64, 0].float()) and float(done["kept"][0, 0, 0]) == 1
    kept = done["kept"]
    del done
    back = ops.gated_recurrence_grad(value, gate, value, kept, torch.ones(1, 1, device="cuda"))
    want = value.clone()
    want[0, -1] += 1
    assert torch.equal(back["value"], want) and not back["gate"].any() and float(back["state"]) == 0


def test_lookup_of_the_most_tokens():
    tokens = torch.arange(MOST, device="cuda", dtype=torch.int32) % 1003 - 1
    table = torch.randn(1000, 1, device="cuda").half()
    got = ops.embedding(table, tokens)
    for first in (0, 1 << 30, MOST - 5000):
        of = tokens[first:first + 5000].long()
        assert torch.equal(got[first:first + 5000], torch.where(((of >= 0) & (of < 1000))[:, None], table[of.clamp(0, 999)], 0)), first
