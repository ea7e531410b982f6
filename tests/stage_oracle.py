"""Plain forms in 64 bits of the stage operators, on the CPU, with bounds on how far a correct 32-bit computation can be off.

A value rounded to a type is off by at most half a step, ``half_step`` times its size.  U is that of 32 bits.  Bounds are sums over a
result's terms of what each rounding on its way can add, taken over absolute values, so that cancellation is covered."""
import math

import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# below the smallest normal number a type's steps stop shrinking
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def rounded(value, bound, dtype):
    """The bound of `value`, known to `bound`, after one rounding to dtype."""
    return bound + HALF_STEP[dtype] * (value.abs() + bound) + SMALLEST[dtype]


def assert_near(got, want, bound, what=""):
    assert tuple(got.shape) == tuple(want.shape), (what, got.shape, want.shape)
    got = got.detach().double().cpu()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | ((got - want).abs() <= bound))
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} too far off, first at {at}: {got[at].item()!r}, "
                             f"expected {want[at].item()!r} within {(bound[at] if torch.is_tensor(bound) else bound)!r}")


# ---- embedding -------------------------------------------------------------------------------------------------------

def embedding(table, tokens, scale):
    t = table.double()
    tokens = tokens.long()
    real = (tokens >= 0) & (tokens < len(t))
    want = (t[tokens.clamp(0, max(len(t) - 1, 0))] if len(t) else torch.zeros(*tokens.shape, t.shape[1], dtype=torch.float64)) * scale
    want = torch.where(real[..., None], want, torch.zeros((), dtype=torch.float64))
    return want, rounded(want, U * want.abs(), table.dtype)


def embedding_grad(grad, tokens, rows, scale, out_dtype, old=None):
    """A row of n occurrences: n additions, a product and, with `old`, one more addition."""
    g, tokens = grad.double().reshape(-1, grad.shape[-1]), tokens.long().reshape(-1)
    real = (tokens >= 0) & (tokens < rows)
    g, tokens = g[real], tokens[real]
    total = torch.zeros(rows, g.shape[1], dtype=torch.float64).index_add_(0, tokens, g)
    size = torch.zeros_like(total).index_add_(0, tokens, g.abs())
    count = torch.bincount(tokens, minlength=rows)[:, None].double()
    want, bound = total * scale, (count + 2) * U * size * abs(scale)
    if old is not None:
        want = want + old.double()
        bound = bound + U * (size * abs(scale) + old.double().abs())
    return want, rounded(want, bound, out_dtype)


# ---- gated linear recurrence -----------------------------------------------------------------------------------------

def _gates(gate):
    """sigmoid(gate), 1 - sigmoid(gate), and a bound on what a step's factors are off by relative to the smaller one: exp's argument is
    rounded once (and so is the constant in it), exp, the addition, the reciprocal and the product once more or a full step; the larger one is one rounding of 1
    less the smaller."""
    g = gate.double()
    a, b = torch.sigmoid(g), torch.sigmoid(-g)
    off = (3 * g.abs() + 10) * U
    small = torch.minimum(a, b)
    return a, b, torch.where(a < b, a * off, small * off + U), torch.where(b < a, b * off, small * off + U)


def recurrence(gate, value, state, lengths):
    """(out, final state, states in front of each step, their bounds): a step h = a h + b v in 32 bits adds its rounding and what a and b are off by; the composition
    of runs rounds every product and sum of a step again, at most three times (its run, its block, its segment)."""
    n, steps, width = value.shape
    a, b, off_a, off_b = _gates(gate)
    v = value.double()
    h = torch.zeros(n, width, dtype=torch.float64) if state is None else state.double()
    e = torch.zeros_like(h)
    ends = torch.full((n,), steps) if lengths is None else lengths.long().clamp(0, steps)
    out, bound, before, before_bound = [], [], [], []
    for t in range(steps):
        before.append(h)
        before_bound.append(e)
        live = (ends > t)[:, None]
        new = a[:, t] * h + b[:, t] * v[:, t]
        size = a[:, t] * h.abs() + b[:, t] * v[:, t].abs()
        new_e = a[:, t] * e + off_a[:, t] * (h.abs() + e) + off_b[:, t] * v[:, t].abs() + 10 * U * (size + a[:, t] * e)
        h, e = torch.where(live, new, h), torch.where(live, new_e, e)
        out.append(torch.where(live, h, 0))
        bound.append(torch.where(live, e, 0))
    stack = lambda x: torch.stack(x, 1) if x else torch.zeros(n, 0, width, dtype=torch.float64)  # noqa: E731
    return stack(out), stack(bound), h, e, stack(before), stack(before_bound)


def recurrence_grad(grad, gate, value, grad_state, lengths, before, before_bound):
    n, steps, width = value.shape
    a, b, off_a, off_b = _gates(gate)
    v, g = value.double(), grad.double()
    ends = torch.full((n,), steps) if lengths is None else lengths.long().clamp(0, steps)
    d = torch.zeros(n, width, dtype=torch.float64) if grad_state is None else grad_state.double()
    e = torch.zeros_like(d)
    d_gate, d_value, e_gate, e_value = (torch.zeros(n, steps, width, dtype=torch.float64) for _ in range(4))
    for t in reversed(range(steps)):
        live = (ends > t)[:, None]
        now = g[:, t] + d
        now_e = e + 10 * U * (g[:, t].abs() + d.abs() + e)
        far = before[:, t] - v[:, t]
        far_e = before_bound[:, t] + U * (before[:, t].abs() + v[:, t].abs())
        d_value[:, t] = torch.where(live, b[:, t] * now, 0)
        e_value[:, t] = torch.where(live, b[:, t] * now_e + off_b[:, t] * (now.abs() + now_e) + U * (b[:, t] * now).abs(), 0)
        p = a[:, t] * b[:, t]
        p_e = off_a[:, t] * b[:, t] + off_b[:, t] * a[:, t] + off_a[:, t] * off_b[:, t] + 2 * U * p
        d_gate[:, t] = torch.where(live, now * far * p, 0)
        e_gate[:, t] = torch.where(live, now_e * (far.abs() + far_e) * (p + p_e) + now.abs() * (far_e * (p + p_e) + far.abs() * p_e) + 3 * U * (now * far * p).abs(), 0)
        d = torch.where(live, a[:, t] * now, d)
        e = torch.where(live, a[:, t] * now_e + off_a[:, t] * (now.abs() + now_e) + U * (a[:, t] * now).abs(), e)
    return d_gate, e_gate, d_value, e_value, d, e


# ---- gated feed-forward block ----------------------------------------------------------------------------------------

def _product(a, b, a_bound=None, b_bound=None):
    """a @ b and its bound: every product rounded (exact for 16-bit factors, as a matrix instruction adds them in any order) and k additions in 32 bits."""
    size = a.abs() @ b.abs()
    bound = (a.shape[1] + 4) * U * size
    if a_bound is not None:
        bound = bound + a_bound @ b.abs()
    if b_bound is not None:
        bound = bound + a.abs() @ b_bound + (a_bound @ b_bound if a_bound is not None else 0)
    return a @ b, bound


def activation(g, name):
    """Value, slope, and a bound of the slope's own slope."""
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p)), 0.6
    if name == "gelu":
        root = math.sqrt(2 / math.pi)
        t = torch.tanh(root * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * root * (1 + 3 * 0.044715 * g * g), 1.2
    return g.clamp(min=0), (g > 0).double(), 0.0


def ffn(x, w_in, w_out, name, grad=None):
    """dict of (value, bound) for out, x, w_in, w_out: the operator rounds hidden, and for the gradients d_pre, to the type, and keeps g and u in 24 bits
    (15 behind the first: off by 2^-16 at most)."""
    dtype = x.dtype
    hidden = w_in.shape[0] // 2
    x, w_in, w_out = x.double(), w_in.double(), w_out.double()
    pre, pre_e = _product(x, w_in.t())
    (g, u), (g_e, u_e) = pre.split(hidden, 1), pre_e.split(hidden, 1)
    act, slope, bend = activation(g, name)
    steep = 1.2   # (the largest slope)
    act_e = steep * g_e + 16 * U * (g.abs() + act.abs())   # (exp of |g| rounds its argument: a relative error of |g| U, times act; |g act'| <= 1.2 |g|)
    act_e = act_e + 2 * U * g.abs() * g.abs().clamp(max=20) * torch.exp(-g.abs().clamp(max=20))
    h = act * u
    h_e = rounded(h, act_e * u.abs() + act.abs() * u_e + act_e * u_e + U * h.abs(), dtype)
    y, y_e = _product(h, w_out.t(), h_e)
    found = dict(out=(y, rounded(y, y_e, dtype)))
    if grad is None:
        return found
    d_y = grad.double()
    d_h, d_h_e = _product(d_y, w_out)
    # from g and u as kept
    gk_e, uk_e = (e + 2.0 ** -16 * (v.abs() + e) for v, e in ((g, g_e), (u, u_e)))
    slope_e = bend * gk_e + 40 * U + (0.0 if name != "relu" else (g.abs() <= gk_e).double())
    actk_e = steep * gk_e + 40 * U * (g.abs() + 1)
    def three(a, a_e, b, b_e, c, c_e):
        return (a.abs() + a_e) * (b.abs() + b_e) * (c.abs() + c_e) - (a * b * c).abs() + 3 * U * (a * b * c).abs()
    one, zero = torch.ones_like(g), torch.zeros_like(g)
    d_g, d_u = d_h * u * slope, d_h * act
    d_g_e, d_u_e = three(d_h, d_h_e, u, uk_e, slope, slope_e), three(d_h, d_h_e, act, actk_e, one, zero)
    d_pre = torch.cat([d_g, d_u], 1)
    d_pre_e = rounded(d_pre, torch.cat([d_g_e, d_u_e], 1), dtype)
    h_e = rounded(h, actk_e * u.abs() + act.abs() * uk_e + actk_e * uk_e + U * h.abs(), dtype)   # (of the hidden made again from them)
    for key, (value, bound) in dict(x=_product(d_pre, w_in, d_pre_e), w_in=_product(d_pre.t(), x, d_pre_e.t()),
                                    w_out=_product(d_y.t(), h, None, h_e)).items():
        found[key] = (value, bound)   # (the caller rounds to the output's type)
    return found


# ---- log probabilities -----------------------------------------------------------------------------------------------

def logprobs(logits, tokens, k):
    """(logprob, entropy, every log probability, ids, their log probabilities).  NaN rows as documented."""
    x, tokens = logits.double().cpu(), tokens.long().cpu()
    n, vocab = x.shape
    wrong = (torch.isnan(x) | (x == math.inf)).any(1)
    empty = (x == -math.inf).all(1)
    every = torch.log_softmax(torch.where((wrong | empty)[:, None], torch.zeros_like(x), x), 1)
    every = torch.where(empty[:, None], torch.full_like(x, -math.inf), every)
    p = torch.exp(every)
    entropy = -torch.where(p > 0, p * every, 0).sum(1)
    real = (tokens >= 0) & (tokens < vocab)
    lp = torch.where(real, every.gather(1, tokens.clamp(0, vocab - 1)[:, None])[:, 0], 0)
    nan = torch.full((), math.nan, dtype=torch.float64)
    lp, entropy = torch.where(wrong, nan, lp), torch.where(wrong, nan, entropy)
    key = torch.where(torch.isnan(x), torch.zeros_like(x), x)
    best, ids = torch.sort(key, dim=1, descending=True, stable=True)
    m = min(k, vocab)
    ids = torch.where((best[:, :m] == -math.inf) | wrong[:, None], -1, ids[:, :m])
    alts = torch.where(ids < 0, torch.full_like(best[:, :m], -math.inf), every.gather(1, ids.clamp(min=0)))
    alts = torch.where(wrong[:, None], nan, alts)
    if m < k:
        ids = torch.cat([ids, torch.full((n, k - m), -1)], 1)
        alts = torch.cat([alts, torch.where(wrong[:, None], nan, torch.full((n, k - m), -math.inf, dtype=torch.float64))], 1)
    return lp, entropy, every, ids, alts


def logprob_bound(logits):
    """Bounds of log s and of a log probability on top of that, absolute.  A term of the sum has exp's error, 3 U |x - m| + 4 U (times the term: |d| e^d < 0.4, so
    under 6 U each), and at most as many additions on its way as a lane has terms, with the sums of lanes, wavefronts and parts behind (64 more)."""
    vocab = logits.shape[1]
    depth = -(-vocab // 256) * 2 + 64
    return (depth + 8) * U


def logprobs_grad(logits, tokens, every, entropy, gl, ge, dtype):
    x, tokens = logits.double().cpu(), tokens.long().cpu()
    n, vocab = x.shape
    real = (tokens >= 0) & (tokens < vocab)
    gl = torch.where(real, gl.double().cpu() if gl is not None else torch.zeros(n, dtype=torch.float64), 0)[:, None]
    ge = (ge.double().cpu() if ge is not None else torch.zeros(n, dtype=torch.float64))[:, None]
    p = torch.exp(every)
    one = torch.zeros_like(x).scatter_(1, tokens.clamp(0, vocab - 1)[:, None], 1)
    lp = torch.where(p > 0, every, 0)
    d = gl * (one - p) - ge * p * (lp + entropy[:, None])
    empty = (x == -math.inf).all(1)
    d = torch.where(empty[:, None], torch.zeros_like(d), d)
    off = logprob_bound(logits) + U * 4 * (lp.abs() + 8)                       # of log p, absolute, and so of p, relative
    far = lp.abs() + entropy.abs()[:, None] + 1
    bound = p * (off * 2 * (gl.abs() + ge.abs() * far) + ge.abs() * (off + logprob_bound(logits) * (math.log(vocab) + 2) * 2)) + 4 * U * (gl.abs() * (one + p) + ge.abs() * p * far)
    bound = bound.nan_to_num(nan=0.0)
    return d, rounded(d.nan_to_num(nan=0.0), bound, dtype)
