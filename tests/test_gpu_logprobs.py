"""Token log probabilities, entropy, alternatives and their gradient against the plain forms in 64 bits."""
import math

import pytest
import torch

import paper_2510_05112_amd as fp
import stage_oracle as oracle

pytestmark = pytest.mark.gpu
ops = fp.stage_ops
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def inputs(n, vocab, dtype, seed=0, masked=0.0):
    g = torch.Generator().manual_seed(seed + n + vocab)
    logits = (3 * torch.randn(n, vocab, generator=g)).to(dtype)
    if masked:
        logits[torch.rand(n, vocab, generator=g) < masked] = -math.inf
    return logits, torch.randint(0, vocab, (n,), generator=g), torch.randn(n, generator=g), torch.randn(n, generator=g)


def check(logits, tokens, k, gl=None, ge=None, on_gpu=None, what=""):
    vocab = logits.shape[1]
    lp, entropy, every, ids, alts = oracle.logprobs(logits, tokens, k)
    d_logits = logits.cuda() if on_gpu is None else on_gpu
    done = ops.token_logprobs(d_logits, tokens.cuda(), k)
    off = oracle.logprob_bound(logits)
    finite = lambda t: t.nan_to_num(nan=0.0, posinf=0.0, neginf=0.0).abs()  # noqa: E731
    oracle.assert_near(done["logprob"], lp, off + 4 * oracle.U * finite(lp), what + " logprob")
    # log s and w / s: the second is a mean of d, its terms off by exp's error and theirs
    oracle.assert_near(done["entropy"], entropy, 2 * off * (math.log(vocab) + 2 + finite(entropy)), what + " entropy")
    if k:
        assert torch.equal(done["ids"].cpu().long(), ids), what + " ids"
        oracle.assert_near(done["logprobs"], alts, off + 4 * oracle.U * finite(alts), what + " alternatives")
    if gl is not None or ge is not None:
        want, bound = oracle.logprobs_grad(logits, tokens, every, entropy, gl, ge, logits.dtype)
        on = [None if t is None else t.cuda() for t in (gl, ge)]
        got = ops.token_logprobs_grad(d_logits, tokens.cuda(), done["lse"], done["entropy"], *on)
        oracle.assert_near(got, want, bound, what + " gradient")
        again = d_logits.clone()
        ops.token_logprobs_grad(again, tokens.cuda(), done["lse"], done["entropy"], *on, out=again)
        assert torch.allclose(again, got, rtol=0, atol=0, equal_nan=True)   # (a row that is no number is not equal to itself)
    return done


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,vocab,k", [(1, 1, 1), (1, 1, 0), (3, 2, 4), (5, 7, 0), (2, 63, 32), (61, 1000, 8), (1, 4096, 1), (2, 4097, 5), (3, 16384, 20), (2, 16385, 32), (4, 50001, 3),
                                       (1, 131077, 17), (1, 300000, 0), (1100, 300, 2), (1030, 40, 0)])
def test_sizes(dtype, n, vocab, k):
    logits, tokens, gl, ge = inputs(n, vocab, dtype)
    check(logits, tokens, k, gl, ge)
    check(logits, tokens.int(), k, gl, None)
    check(logits, tokens, k, None, ge)


@pytest.mark.parametrize("dtype", TYPES)
def test_masks(dtype):
    for vocab, k in ((50, 9), (5000, 7), (40000, 6)):
        logits, tokens, gl, ge = inputs(9, vocab, dtype, 1, masked=0.95)
        logits[1] = -math.inf                                    # nothing left
        logits[2] = -math.inf                                    # one left, not the token
        logits[2, (tokens[2] + 1) % vocab] = 2.0
        logits[3] = -math.inf                                    # one left, the token: certain
        logits[3, tokens[3]] = -5.0
        logits[4] = torch.finfo(dtype).min                       # masks of the type's lowest value
        logits[4, :3] = 1.0
        logits[5] = torch.finfo(dtype).min                       # in all places
        tokens[6], tokens[7] = -1, vocab                         # paddings
        done = check(logits, tokens, k, gl, ge)
        assert float(done["logprob"][3]) == 0 and float(done["entropy"][3]) == 0 and float(done["logprob"][6]) == 0


def test_rows_with_nan_or_infinity():
    logits, tokens, gl, ge = inputs(6, 9000, torch.float32, 2)
    logits[1, 5], logits[2, 8999], logits[4] = math.nan, math.inf, math.nan
    check(logits, tokens, 4)
    done = ops.token_logprobs(logits.cuda(), tokens.cuda(), 4)
    got = ops.token_logprobs_grad(logits.cuda(), tokens.cuda(), done["lse"], done["entropy"], gl.cuda(), ge.cuda()).cpu()
    assert torch.isnan(got[[1, 2, 4]]).all() and torch.isfinite(got[[0, 3, 5]]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits_come_by_ascending_id(dtype):
    for vocab in (100, 5000, 40000):
        check(torch.zeros(3, vocab).to(dtype), torch.zeros(3, dtype=torch.int64), 20)
        g = torch.Generator().manual_seed(vocab)
        few = torch.randint(-1, 3, (5, vocab), generator=g).to(dtype)
        few[0, ::2] = -0.0                                       # equal to 0
        check(few, torch.full((5,), vocab - 1), 32)


@pytest.mark.parametrize("dtype", TYPES)
def test_extreme_logits(dtype):
    most = torch.finfo(dtype).max
    for vocab in (64, 9000):
        logits, tokens, gl, ge = inputs(4, vocab, dtype, 3)
        logits[0, 7], logits[0, 9] = most, -most                 # one takes all
        logits[1] = most
        logits[2] = -most
        logits[3] += 100.0
        check(logits, tokens, 5, gl, ge)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_apart_and_at_any_address(dtype):
    n, vocab = 7, 5003
    logits, tokens, gl, ge = inputs(n, vocab, dtype, 4)
    for first, width in ((0, vocab), (0, 5016), (1, 5016), (3, 5011), (8, 5016)):
        wide = torch.full((n, width + (first > 0) * 13), math.nan).to(dtype).cuda()
        wide[:, first:first + vocab] = logits.cuda()
        check(logits, tokens, 6, gl, ge, wide[:, first:first + vocab], f"{first} of {width}")
        done = ops.token_logprobs(logits.cuda(), tokens.cuda())
        before = wide.clone()
        ops.token_logprobs_grad(wide[:, first:first + vocab], tokens.cuda(), done["lse"], done["entropy"], gl.cuda(), out=wide[:, first:first + vocab])
        assert torch.equal(wide[:, :first].isnan(), before[:, :first].isnan()) and wide[:, first + vocab:].isnan().all()


def test_gradients_against_differences():
    logits, tokens, gl, ge = inputs(3, 11, torch.float32, 5)
    done = ops.token_logprobs(logits.cuda(), tokens.cuda())
    got = ops.token_logprobs_grad(logits.cuda(), tokens.cuda(), done["lse"], done["entropy"], gl.cuda(), ge.cuda()).cpu()

    def total(x):
        lp, entropy, *_ = oracle.logprobs(x, tokens, 0)
        return float((lp * gl.double()).sum() + (entropy * ge.double()).sum())

    step = 1e-4
    for i in range(33):
        up, down = logits.double().clone(), logits.double().clone()
        up.reshape(-1)[i] += step
        down.reshape(-1)[i] -= step
        want = (total(up) - total(down)) / (2 * step)
        # (step^2 / 6 times a third derivative, of size |log p| and less: under 100; the operator's own error is some 1e-6 of its terms)
        assert abs(float(got.reshape(-1)[i]) - want) <= 5e-6 + 1e-5 * abs(want)


def test_no_rows():
    logits = torch.empty(0, 100, device="cuda")
    tokens = torch.empty(0, dtype=torch.int64, device="cuda")
    done = ops.token_logprobs(logits, tokens, 3)
    assert done["ids"].shape == (0, 3)
    assert ops.token_logprobs_grad(logits, tokens, done["lse"], done["entropy"]).shape == (0, 100)


def test_more_than_2_to_the_32_logits():
    n, vocab = 33000, 131072
    logits = torch.zeros(n, vocab, dtype=torch.bfloat16, device="cuda")
    logits[n - 1, vocab - 1] = 20.0
    tokens = torch.full((n,), vocab - 1, device="cuda")
    done = ops.token_logprobs(logits, tokens, 1)
    want = oracle.logprobs(logits[-1:].cpu(), tokens[-1:].cpu(), 1)
    assert int(done["ids"][n - 1, 0]) == vocab - 1 and int(done["ids"][n - 2, 0]) == 0
    assert abs(float(done["logprob"][n - 1]) - float(want[0])) < 1e-5
    ops.token_logprobs_grad(logits, tokens, done["lse"], done["entropy"], torch.ones(n, device="cuda"), out=logits)
    p = math.exp(float(want[0]))
    assert abs(float(logits[n - 1, vocab - 1]) - (1 - p)) <= 2 ** -8 * (1 - p) + 1e-6


@pytest.mark.parametrize("vocab,k", [(2, 0), (3, 2)])
def test_more_rows_than_a_grid_has_workgroups(vocab, k):
    # (a workgroup looks at a row, and a grid has 2^24 - 1 of them)
    n = (1 << 24) + 83
    rows = torch.randn(1000, vocab, device="cuda").bfloat16()
    logits = rows.repeat(n // 1000 + 1, 1)[:n]
    tokens = torch.full((n,), vocab - 1, device="cuda", dtype=torch.int32)
    gl = torch.ones(n, device="cuda")
    want, want_tokens = ops.token_logprobs(rows, tokens[:1000], k), tokens[:1000]
    want_grad = ops.token_logprobs_grad(rows, want_tokens, want["lse"], want["entropy"], gl[:1000])
    done = ops.token_logprobs(logits, tokens, k)
    got = ops.token_logprobs_grad(logits, tokens, done["lse"], done["entropy"], gl, out=logits)
    for first in (0, (n - 100) // 1000 * 1000):
        of = slice(first, min(first + 1000, n))
        for name, t in done.items():
            assert torch.equal(t[of], want[name][:of.stop - first]), (name, first)
        assert torch.equal(got[of], want_grad[:of.stop - first]), first


@pytest.mark.parametrize("vocab", [300, 700, 2003, 16384, 40001, 262144])
def test_alternatives_of_logits_in_any_order(vocab):
    # (ascending, descending, of one value, of one value but for a few, few values with the largest at the end, masked but for few)
    at = torch.arange(vocab)
    rows = torch.stack([at * (9.0 / vocab), 5 - at * (9.0 / vocab), torch.full((vocab,), -2.5), torch.where(at % 677 == 3, 1.0, 0.5), (at > vocab - 600).float() + (at > vocab - 5).float(),
                        torch.where(at % 97 == 5, at * (1.0 / vocab), -math.inf), torch.where(at % 301 == 0, -math.inf, -3.0), torch.where(at < 10, at * 1.0, torch.finfo(torch.float32).min)])
    tokens = torch.full((len(rows),), vocab - 1)
    for dtype in TYPES:
        for k in (1, 7, 32):
            check(rows.clamp(min=torch.finfo(dtype).min).where(rows > -math.inf, rows).to(dtype), tokens, k, what=f"{dtype} {k}")


def test_alternatives_of_many_parts():
    # (one row in a thousand parts: the largest logits in any of them; the last row has them in parts of which a lane takes several)
    vocab = 4_500_000
    at = torch.arange(vocab)
    block = at // 4416 % 256
    rows = torch.stack([torch.randn(vocab), torch.zeros(vocab), at * 1e-6, at * -1e-6, torch.where(block < 31, 5.0, torch.where(block == 31, 1.0, 0.0))])
    for row in rows:
        for k in (1, 8, 32):
            check(row[None], torch.tensor([vocab - 1]), k, what=str(k))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_rows(dtype):
    # (rows that one wavefront takes, with masks, equal logits and odd addresses)
    for vocab, k in ((1, 1), (7, 4), (511, 32), (2000, 8), (4096, 32), (4097, 3)):
        logits, tokens, gl, ge = inputs(600, vocab, dtype, 6, masked=0.2 if vocab > 1 else 0.0)
        logits[5] = 1.0
        logits[6] = -math.inf
        logits[7, vocab // 2] = math.nan
        logits[8] = torch.where(torch.arange(vocab) % 3 == 0, -2.0, 0.25)
        check(logits, tokens, k, gl, ge)
        wide = torch.zeros(600, vocab + 3, device="cuda").to(dtype)
        wide[:, 1:vocab + 1] = logits.cuda()
        check(logits, tokens, k, gl, None, wide[:, 1:vocab + 1], str(vocab))
