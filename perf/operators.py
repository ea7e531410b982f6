"""The operators of a language model's pipeline stages, as cases that can be timed.

A case is one pass through one operator as a stage's items call it: the embedding of the first stage (``embedding``),
the gated recurrence that mixes tokens (``recurrence``), the gated feed-forward block (``ffn``) and the log
probabilities of the last stage (``logprobs``), forward alone as in serving or with the gradients as in training.
``listed`` names the cases, ``draw`` gives more of the same ranges, ``prepare`` makes what a program has in hand
before the call, ``run`` is the call: in plain torch operations, or with ``own`` through the framework's operators.
"""
from __future__ import annotations

import math

import numpy as np
import torch

#: False: ``run`` computes the plain form; True: it calls the framework's operators.
own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # a serving step of a few dozen requests looks its tokens up: nothing but latency
        dict(name="embedding_step", op="embedding", pass_="forward", tokens=61, vocab=65536, width=2560, type="bf16"),
        # the weight-gradient item of the first stage, four sequences of a micro-batch, padding at their ends
        dict(name="embedding_gradient", op="embedding", pass_="gradient", tokens=4096, vocab=65536, width=4096, type="bf16"),
        # the same under the large vocabulary that makes the first stage the heavy one
        dict(name="embedding_gradient_large", op="embedding", pass_="gradient", tokens=16384, vocab=262144, width=2560, type="bf16"),
        # one token for each of a few dozen requests, the states carried from step to step
        dict(name="recurrence_step", op="recurrence", pass_="forward", batch=61, steps=1, width=2560, type="bf16", ragged=False),
        # forward and backward items of a micro-batch with sequences of unequal length
        dict(name="recurrence_train", op="recurrence", pass_="train", batch=4, steps=1021, width=4096, type="bf16", ragged=True),
        # one long prompt: no batch to be parallel over
        dict(name="recurrence_long", op="recurrence", pass_="forward", batch=1, steps=65536, width=2560, type="f16", ragged=False),
        # a serving step: as many bytes of weights as of a training step, five rows
        dict(name="ffn_step", op="ffn", pass_="forward", tokens=5, width=4096, hidden=10752, act="silu", type="bf16"),
        # F, B and W items of a small micro-batch, its length no multiple of anything
        dict(name="ffn_train_small", op="ffn", pass_="train", tokens=509, width=2560, hidden=6912, act="gelu", type="f16"),
        # F, B and W items of a large micro-batch
        dict(name="ffn_train", op="ffn", pass_="train", tokens=8192, width=4096, hidden=10752, act="silu", type="bf16"),
        # the answers of a serving step, with the eight likeliest tokens of each
        dict(name="logprobs_step", op="logprobs", pass_="forward", rows=61, vocab=262144, alternatives=8, masked=False, type="bf16"),
        # loss, entropy and their gradient on the last stage
        dict(name="logprobs_train", op="logprobs", pass_="train", rows=4096, vocab=65536, alternatives=0, masked=False, type="bf16"),
        # a grammar's mask forbids most tokens, in one row all of them; rows that begin at odd addresses
        dict(name="logprobs_masked", op="logprobs", pass_="forward", rows=509, vocab=100003, alternatives=5, masked=True, type="f16"),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["embedding", "recurrence", "ffn", "logprobs"])
    kind = rng.choice(["bf16", "f16"])
    if op == "embedding":
        return dict(op=op, pass_=rng.choice(["forward", "gradient"]), tokens=_spread(rng, 1, 32768), vocab=_spread(rng, 1000, 200000),
                    width=_spread(rng, 33, 4096), type=rng.choice(["bf16", "f16", "f32"]))
    if op == "recurrence":
        batch, steps = _spread(rng, 1, 64), _spread(rng, 1, 32768)
        return dict(op=op, pass_=rng.choice(["forward", "train"]), batch=batch, steps=min(steps, 65536 // batch), width=_spread(rng, 33, 4096),
                    type=rng.choice(["bf16", "f16", "f32"]), ragged=rng.random() < 0.5)
    if op == "ffn":
        width = 8 * _spread(rng, 32, 512)
        return dict(op=op, pass_=rng.choice(["forward", "train"]), tokens=_spread(rng, 1, 8192), width=width, hidden=8 * (width * rng.randint(16, 21) // 64),
                    act=rng.choice(["silu", "gelu"]), type=kind)
    vocab = _spread(rng, 1000, 300000)
    rows = min(_spread(rng, 1, 4096), 268435456 // vocab)
    train = rng.random() < 0.5
    return dict(op=op, pass_="train" if train else "forward", rows=rows, vocab=vocab, alternatives=0 if train else rng.randint(0, 20),
                masked=rng.random() < 0.3, type=rng.choice(["bf16", "f16", "f32"]))


def work(case):
    size = _SIZES[case["type"]]
    if case["op"] == "embedding":
        rows = case["tokens"] * 2 if case["pass_"] == "forward" else case["tokens"] + case["vocab"]
        return {"bytes": rows * case["width"] * size + 4 * case["tokens"], "flops": case["tokens"] * case["width"]}
    if case["op"] == "recurrence":
        n, state = case["batch"] * case["steps"] * case["width"], 4 * case["batch"] * case["width"]
        train = case["pass_"] == "train"
        return {"bytes": (6 if train else 3) * n * size + (4 if train else 2) * state, "flops": (24 if train else 8) * n}
    if case["op"] == "ffn":
        t, k, f = case["tokens"], case["width"], case["hidden"]
        train = case["pass_"] == "train"
        return {"bytes": size * ((4 if train else 2) * t * k + (6 if train else 3) * f * k), "flops": (18 if train else 6) * t * k * f}
    n = case["rows"] * case["vocab"]
    train = case["pass_"] == "train"
    return {"bytes": n * size * (2 if train else 1) + case["rows"] * (24 if train else 16 + 8 * case["alternatives"]), "flops": (10 if train else 6) * n}


def _tokens(n, vocab, gen):
    """Token ids as a text has them: a few make up much of it (rank r with about 1 / r), spread over the vocabulary."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = torch.floor(torch.exp(u * math.log(vocab))).long().clamp_(1, vocab) - 1
    return ((rank * 7919) % vocab).int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = _TYPES[case["type"]]

    def normal(*shape, scale=1.0, type_=kind):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(type_)

    if case["op"] == "embedding":
        tokens = _tokens(case["tokens"], case["vocab"], gen)
        # (padding at the end of every sequence: token -1)
        position = torch.arange(case["tokens"], device="cuda") % 1024
        tokens = torch.where(position >= 1000, torch.full_like(tokens, -1), tokens)
        rows = case["vocab"] if case["pass_"] == "forward" else case["tokens"]
        return dict(case, tokens=tokens, scale=math.sqrt(case["width"]), data=normal(rows, case["width"], scale=0.02))
    if case["op"] == "recurrence":
        b, t, c = case["batch"], case["steps"], case["width"]
        # (gates that keep most of a state: it lasts for tens of steps, in some channels for thousands)
        gate = normal(b, t, c, type_=torch.float32).add_(torch.linspace(0, 7, c, device="cuda")).to(kind)
        lengths = torch.randint(0, t + 1, (b,), generator=gen, device="cuda", dtype=torch.int32) if case["ragged"] else None
        if lengths is not None:
            lengths[0] = t
        state = dict(case, gate=gate, value=normal(b, t, c), state=normal(b, c, type_=torch.float32), lengths=lengths)
        if case["pass_"] == "train":
            state.update(grad=normal(b, t, c), grad_state=normal(b, c, type_=torch.float32))
        return state
    if case["op"] == "ffn":
        t, k, f = case["tokens"], case["width"], case["hidden"]
        state = dict(case, x=normal(t, k), w_in=normal(2 * f, k, scale=k ** -0.5), w_out=normal(k, f, scale=f ** -0.5))
        if case["pass_"] == "train":
            state.update(grad=normal(t, k))
        return state
    n, v = case["rows"], case["vocab"]
    tokens = _tokens(n, v, gen)
    logits = normal(n, v, scale=3.0)
    # (the model has learnt something: the given token is ahead of most)
    logits.scatter_add_(1, tokens.long()[:, None], torch.full((n, 1), 9.0, device="cuda", dtype=kind))
    if case["masked"]:
        logits.masked_fill_(torch.rand((n, v), generator=gen, device="cuda") < 0.9, -math.inf)
        logits[n // 2] = -math.inf
    state = dict(case, logits=logits, tokens=tokens)
    if case["pass_"] == "train":
        # (policy-gradient weights for the tokens, a bonus for the entropy)
        state.update(grad_logprob=normal(n, type_=torch.float32), grad_entropy=torch.full((n,), 0.01, device="cuda"))
    return state


def run(state):
    return (_own if own else _plain)[state["op"]](state)


# ---- through the framework's operators -------------------------------------------------------------------------------

def _own_embedding(s):
    from paper_2510_05112_amd import stage_ops
    if s["pass_"] == "forward":
        return stage_ops.embedding(s["data"], s["tokens"], s["scale"])
    return stage_ops.embedding_grad(s["data"], s["tokens"], s["vocab"], s["scale"])


def _own_recurrence(s):
    from paper_2510_05112_amd import stage_ops
    train = s["pass_"] == "train"
    done = stage_ops.gated_recurrence(s["gate"], s["value"], s["state"], s["lengths"], keep=train)
    if not train:
        return [done["out"], done["state"]]
    back = stage_ops.gated_recurrence_grad(s["grad"], s["gate"], s["value"], done["kept"], s["grad_state"], s["lengths"])
    return [done["out"], done["state"], back["gate"], back["value"], back["state"]]


def _own_ffn(s):
    from paper_2510_05112_amd import stage_ops
    train = s["pass_"] == "train"
    done = stage_ops.gated_ffn(s["x"], s["w_in"], s["w_out"], s["act"], keep=train)
    if not train:
        return done["out"]
    back = stage_ops.gated_ffn_input_grad(s["grad"], s["w_in"], s["w_out"], done["kept"], s["act"])
    weights = stage_ops.gated_ffn_weight_grad(s["x"], s["grad"], done["kept"], back["kept"])
    return [done["out"], back["x"], weights["w_in"], weights["w_out"]]


def _own_logprobs(s):
    from paper_2510_05112_amd import stage_ops
    done = stage_ops.token_logprobs(s["logits"], s["tokens"], s["alternatives"])
    found = [done["logprob"], done["entropy"]]
    if s["pass_"] == "train":
        found.append(stage_ops.token_logprobs_grad(s["logits"], s["tokens"], done["lse"], done["entropy"], s["grad_logprob"], s["grad_entropy"]))
    return found + ([done["ids"], done["logprobs"]] if s["alternatives"] else [])


_own = dict(embedding=_own_embedding, recurrence=_own_recurrence, ffn=_own_ffn, logprobs=_own_logprobs)


# ---- plain forms -----------------------------------------------------------------------------------------------------

def _plain_embedding(s):
    data, tokens = s["data"], s["tokens"].long()
    real = tokens >= 0
    if s["pass_"] == "forward":
        return (data[tokens.clamp(min=0)].float() * s["scale"] * real[:, None]).to(data.dtype)
    total = torch.zeros((s["vocab"] + 1, s["width"]), device="cuda")
    total.index_add_(0, torch.where(real, tokens, s["vocab"]), data.float())
    return (total[:-1] * s["scale"]).to(data.dtype)


def _scan(a, b):
    """h[t] = a[t] h[t-1] + b[t] along dimension 1, from h = 0: by doubling, since the sequence has no parallel form of one operation."""
    a, d = a.clone(), 1
    while d < a.shape[1]:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _plain_recurrence(s):
    kind, t = s["value"].dtype, s["steps"]
    a, v = torch.sigmoid(s["gate"].float()), s["value"].float()
    b = (1 - a) * v
    live = None
    if s["lengths"] is not None:
        # behind a sequence's end the state stands still and the output is zero
        live = (torch.arange(t, device="cuda")[None] < s["lengths"][:, None])[..., None]
        a, b = torch.where(live, a, 1), torch.where(live, b, 0)
    start = s["state"][:, None]
    first = torch.cat([b[:, :1] + a[:, :1] * start, b[:, 1:]], 1)
    h = _scan(a, first)
    final = h[:, -1]
    shown = h if live is None else torch.where(live, h, 0)
    if s["pass_"] == "forward":
        return [shown.to(kind), final]
    g = s["grad"].float()
    g = g if live is None else torch.where(live, g, 0)
    g = torch.cat([g[:, :-1], g[:, -1:] + s["grad_state"][:, None]], 1)
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    d = _scan(after.flip(1), g.flip(1)).flip(1)
    before = torch.cat([start, h[:, :-1]], 1)
    d_gate, d_value = d * (before - v) * a * (1 - a), d * (1 - a)
    if live is not None:
        d_gate, d_value = torch.where(live, d_gate, 0), torch.where(live, d_value, 0)
    return [shown.to(kind), final, d_gate.to(kind), d_value.to(kind), d[:, 0] * a[:, 0]]


_ROOT = math.sqrt(2 / math.pi)


def _activation(g, name):
    """The activation and its derivative."""
    if name == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    t = torch.tanh(_ROOT * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * _ROOT * (1 + 3 * 0.044715 * g * g)


def _ffn(s, kind):
    x, w_in, w_out = s["x"].to(kind), s["w_in"].to(kind), s["w_out"].to(kind)
    gate, up = (x @ w_in.t()).split(s["hidden"], 1)
    act, slope = _activation(gate, s["act"])
    h = act * up
    y = h @ w_out.t()
    if s["pass_"] == "forward":
        return [y]
    grad = s["grad"].to(kind)
    d_h = grad @ w_out
    d_pre = torch.cat([d_h * up * slope, d_h * act], 1)
    return [y, d_pre @ w_in, d_pre.t() @ x, grad.t() @ h]


def _plain_ffn(s):
    found = [x.to(s["x"].dtype) for x in _ffn(s, torch.float32)]
    return found[0] if s["pass_"] == "forward" else found


def _plain_logprobs(s):
    x, tokens = s["logits"].float(), s["tokens"].long()
    most = x.max(1, keepdim=True).values
    most = torch.where(most == -math.inf, 0, most)
    e = torch.exp(x - most)
    total = e.sum(1, keepdim=True)
    ln = torch.log(total)
    away = torch.where(e > 0, x - most, 0)
    logprob = ((x - most).gather(1, tokens[:, None]) - ln)[:, 0]
    some = total[:, 0] > 0
    logprob = torch.where(some, logprob, -math.inf)
    p = torch.where(total > 0, e / total, 0)
    entropy = torch.where(some, ln[:, 0] - (p * away).sum(1), 0)
    found = [logprob, entropy]
    if s["pass_"] == "train":
        d = -p * (s["grad_logprob"][:, None] + s["grad_entropy"][:, None] * (away - ln + entropy[:, None]))
        d = torch.where(some[:, None], d, 0)
        d.scatter_add_(1, tokens[:, None], torch.where(some, s["grad_logprob"], 0)[:, None])
        found.append(d.to(s["logits"].dtype))
    if s["alternatives"]:
        best, ids = torch.sort(s["logits"], dim=1, descending=True, stable=True)   # (equal ones: the lowest index first)
        best, ids = best[:, :s["alternatives"]].float(), ids[:, :s["alternatives"]]
        found += [torch.where(best == -math.inf, -1, ids).int(), torch.where(best == -math.inf, -math.inf, best - most - ln)]
    return found


_plain = dict(embedding=_plain_embedding, recurrence=_plain_recurrence, ffn=_plain_ffn, logprobs=_plain_logprobs)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embedding":
        tokens = s["tokens"].cpu().numpy()
        data = s["data"].double().cpu().numpy() * s["scale"] if case["pass_"] == "gradient" else None
        if case["pass_"] == "forward":
            rows = s["data"].double()[s["tokens"].long().clamp(min=0)] * s["scale"]
            rows[s["tokens"] < 0] = 0
            return rows
        order = np.argsort(tokens, kind="stable")
        order = order[tokens[order] >= 0]
        out = torch.zeros((case["vocab"], case["width"]), dtype=torch.float64, device="cuda")
        if len(order):
            ids, first = np.unique(tokens[order], return_index=True)
            out[torch.from_numpy(ids).long().cuda()] = torch.from_numpy(np.add.reduceat(data[order], first, axis=0)).cuda()
        return out
    if case["op"] == "recurrence":
        t = case["steps"]
        a = torch.sigmoid(s["gate"].double())
        v = s["value"].double()
        length = s["lengths"].tolist() if s["lengths"] is not None else [t] * case["batch"]
        h = torch.zeros_like(v)
        now = s["state"].double()
        ends = torch.tensor(length, device="cuda")[:, None]
        before = []
        for i in range(t):
            before.append(now)
            now = torch.where(ends > i, torch.lerp(v[:, i], now, a[:, i]), now)
            h[:, i] = torch.where(ends > i, now, 0)
            if case["pass_"] != "train":
                before.clear()
        if case["pass_"] != "train":
            return [h, now]
        d, d_gate, d_value = s["grad_state"].double(), torch.zeros_like(v), torch.zeros_like(v)
        grad = s["grad"].double()
        for i in reversed(range(t)):
            live = ends > i
            d = torch.where(live, d + grad[:, i], d)
            d_value[:, i] = torch.where(live, d * (1 - a[:, i]), 0)
            d_gate[:, i] = torch.where(live, d * (before[i] - v[:, i]) * a[:, i] * (1 - a[:, i]), 0)
            d = torch.where(live, d * a[:, i], d)
        return [h, now, d_gate, d_value, d]
    if case["op"] == "ffn":
        x, w_in, w_out, f = s["x"].double(), s["w_in"].double(), s["w_out"].double(), case["hidden"]
        gate = torch.matmul(x, w_in[:f].t()).requires_grad_(case["pass_"] == "train")
        up = torch.matmul(x, w_in[f:].t())
        if case["act"] == "silu":
            act = gate / (1 + torch.exp(-gate))
        else:
            act = gate / (1 + torch.exp(-2 * _ROOT * gate * (1 + 0.044715 * gate * gate)))
        y = torch.matmul(act.detach() * up, w_out.t())
        if case["pass_"] == "forward":
            return y
        grad = s["grad"].double()
        d_h = torch.matmul(grad, w_out)
        d_gate, = torch.autograd.grad(act, gate, d_h * up)
        d_up, h = d_h * act.detach(), act.detach() * up
        return [y, d_gate @ w_in[:f] + d_up @ w_in[f:], torch.cat([d_gate.t() @ x, d_up.t() @ x]), grad.t() @ h]
    lp, ent, grads, ids, alts = [], [], [], [], []
    for i in range(0, case["rows"], 256):
        x, tok = s["logits"][i:i + 256].double(), s["tokens"][i:i + 256].long()
        empty = (x == -math.inf).all(1)
        every = torch.where(empty[:, None], -math.inf, torch.log_softmax(x, 1))
        p = torch.exp(every)
        h = -torch.where(p > 0, p * every, 0).sum(1)
        lp.append(every.gather(1, tok[:, None])[:, 0])
        ent.append(h)
        if case["pass_"] == "train":
            gl, ge = s["grad_logprob"][i:i + 256].double()[:, None], s["grad_entropy"][i:i + 256].double()[:, None]
            one = torch.zeros_like(x).scatter_(1, tok[:, None], 1)
            d = gl * (one - p) - ge * torch.where(p > 0, p * (every + h[:, None]), 0)
            grads.append(torch.where(empty[:, None], 0, d))
        if case["alternatives"]:
            alts.append(every.topk(case["alternatives"], 1).values)
    found = [torch.cat(lp), torch.cat(ent)]
    if case["pass_"] == "train":
        found.append(torch.cat(grads))
    if case["alternatives"]:
        found += [None, torch.cat(alts)]
    return found
