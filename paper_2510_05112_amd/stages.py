"""Pipeline stages of a language model whose items run on this GPU, so that the tuner's cost table can be measured.

A stage is a list of layers.  A layer runs three kinds of items, as the schedules have them (paper Section 4, Table 1): ``forward`` (FwdPass),
``input_grad`` (CompInputGrad) and ``weight_grad`` (CompWeightGrad; adds to float32 gradients, micro-batch by micro-batch).  What an item
hands to a later one of the same micro-batch it returns, so that any number of micro-batches can be in flight.  The operators are those of
``stage_ops``; the dense products around them are the library's.  A layer of a user's own needs the same three methods and
``kept_bytes`` need not know of it: everything kept is counted by its tensors."""
from __future__ import annotations

import math

from . import stage_ops


def _normal(shape, std, dtype, device, generator):
    import torch
    return (torch.randn(shape, device=device, generator=generator) * std).to(dtype)


def _add_product(total, a, b):
    """total += a^T b, where total is float32: the products are added to it in 32 bits, without a rounding to their type in between."""
    import torch
    torch.addmm(total, a.t(), b, out_dtype=torch.float32, out=total)


class Layer:
    """weights and grads: dicts of tensors by the same names, the latter float32 and zero until a ``weight_grad``."""

    def __init__(self, **weights):
        import torch
        self.weights = weights
        self.grads = {name: torch.zeros_like(w, dtype=torch.float32) for name, w in weights.items()}


class Embedding(Layer):
    """The first layer of the first stage: tokens [batch][steps] (-1: padding) to rows of the table, scaled by sqrt(width)."""

    def __init__(self, vocab, width, dtype, device="cuda", generator=None):
        super().__init__(table=_normal((vocab, width), width ** -0.5, dtype, device, generator))
        self.scale = math.sqrt(width)

    def forward(self, tokens):
        tokens = tokens.contiguous()   # (a text's tokens but the last are a view)
        return stage_ops.embedding(self.weights["table"], tokens, self.scale), dict(tokens=tokens)

    def input_grad(self, grad, kept):
        return None, dict(grad=grad)

    def weight_grad(self, kept, grad_kept):
        grad = grad_kept["grad"]
        stage_ops.embedding_grad(grad.contiguous(), kept["tokens"], len(self.weights["table"]), self.scale, out=self.grads["table"], accumulate=True)


class Recurrence(Layer):
    """x + the gated linear recurrence of two projections of x, over [batch][steps][width]."""

    def __init__(self, width, dtype, device="cuda", generator=None):
        super().__init__(w=_normal((2 * width, width), width ** -0.5, dtype, device, generator))

    def _halves(self, both):
        width = self.weights["w"].shape[1]
        return both[..., :width], both[..., width:]

    def forward(self, x):
        both = (x.reshape(-1, x.shape[-1]) @ self.weights["w"].t()).view(*x.shape[:-1], len(self.weights["w"]))
        done = stage_ops.gated_recurrence(*self._halves(both), keep=True)
        return x + done["out"], dict(x=x, both=both, states=done["kept"])

    def input_grad(self, grad, kept):
        import torch
        back = stage_ops.gated_recurrence_grad(grad, *self._halves(kept["both"]), kept["states"])
        both = torch.cat([back["gate"], back["value"]], -1)
        return grad + (both.view(-1, both.shape[-1]) @ self.weights["w"]).view(grad.shape), dict(both=both)

    def weight_grad(self, kept, grad_kept):
        width = self.weights["w"].shape[1]
        _add_product(self.grads["w"], grad_kept["both"].reshape(-1, 2 * width), kept["x"].reshape(-1, width))


class FeedForward(Layer):
    """x + the gated feed-forward block of x."""

    def __init__(self, width, hidden, dtype, activation="silu", device="cuda", generator=None):
        super().__init__(w_in=_normal((2 * hidden, width), width ** -0.5, dtype, device, generator),
                         w_out=_normal((width, hidden), hidden ** -0.5, dtype, device, generator))
        self.activation = activation

    def forward(self, x):
        rows = x.reshape(-1, x.shape[-1])
        done = stage_ops.gated_ffn(rows, self.weights["w_in"], self.weights["w_out"], self.activation, keep=True)
        return x + done["out"].view(x.shape), dict(x=rows, **done["kept"])

    def input_grad(self, grad, kept):
        rows = grad.reshape(-1, grad.shape[-1])
        back = stage_ops.gated_ffn_input_grad(rows, self.weights["w_in"], self.weights["w_out"], kept, self.activation)
        return grad + back["x"].view(grad.shape), dict(grad=rows, **back["kept"])

    def weight_grad(self, kept, grad_kept):
        stage_ops.gated_ffn_weight_grad(kept["x"], grad_kept["grad"], kept, grad_kept, out=self.grads, accumulate=True)


class Head(Layer):
    """The last layer of the last stage: logits and the log probabilities of given tokens.  The loss is minus the mean of those over the tokens of
    the vocabulary (others are padding), less ``entropy_bonus`` times the mean entropy of those rows."""

    def __init__(self, vocab, width, dtype, entropy_bonus=0.0, device="cuda", generator=None):
        super().__init__(w=_normal((vocab, width), width ** -0.5, dtype, device, generator))
        self.entropy_bonus = entropy_bonus

    def forward(self, x, tokens):
        rows, tokens = x.reshape(-1, x.shape[-1]), tokens.reshape(-1)
        logits = rows @ self.weights["w"].t()
        done = stage_ops.token_logprobs(logits, tokens)
        share = ((tokens >= 0) & (tokens < logits.shape[1])).float()
        share /= share.sum().clamp(min=1)
        loss = -(share * (done["logprob"] + self.entropy_bonus * done["entropy"])).sum()
        return loss, dict(x=rows, shape=x.shape, logits=logits, tokens=tokens, share=share, lse=done["lse"], entropy=done["entropy"])

    def input_grad(self, grad, kept):
        """grad: that of the loss (a number).  The logits' memory becomes their gradient's."""
        g = kept["share"] * -grad
        d = stage_ops.token_logprobs_grad(kept["logits"], kept["tokens"], kept["lse"], kept["entropy"], g, self.entropy_bonus * g if self.entropy_bonus else None,
                                          out=kept["logits"])
        return (d @ self.weights["w"]).view(kept["shape"]), dict(logits=d)

    def weight_grad(self, kept, grad_kept):
        _add_product(self.grads["w"], grad_kept["logits"], kept["x"])


class Stage:
    """Layers in a row.  ``forward`` returns what goes to the next stage and what this one keeps; ``tokens`` is for a ``Head``."""

    def __init__(self, layers):
        self.layers = list(layers)

    def forward(self, x, tokens=None):
        kept = []
        for layer in self.layers:
            x, k = layer.forward(x, tokens) if isinstance(layer, Head) else layer.forward(x)
            kept.append(k)
        return x, kept

    def input_grad(self, grad, kept):
        grad_kept = []
        for layer, k in zip(reversed(self.layers), reversed(kept)):
            grad, g = layer.input_grad(grad, k)
            grad_kept.append(g)
        return grad, grad_kept[::-1]

    def weight_grad(self, kept, grad_kept):
        for layer, k, g in zip(self.layers, kept, grad_kept):
            layer.weight_grad(k, g)


def kept_bytes(kept) -> int:
    """Bytes of device memory behind the tensors in nested lists and dicts, each piece of memory once."""
    import torch
    found, todo = {}, [kept]
    while todo:
        x = todo.pop()
        if isinstance(x, torch.Tensor):
            storage = x.untyped_storage()
            found[storage.data_ptr()] = storage.nbytes()
        elif isinstance(x, dict):
            todo += x.values()
        elif isinstance(x, (list, tuple)) and not isinstance(x, torch.Size):
            todo += x
    return sum(found.values())


def language_model(n_stages: int, layers: int, width: int, hidden: int, vocab: int, dtype=None, device="cuda", seed: int = 0):
    """The stages of a model of `layers` pairs of a recurrence and a feed-forward block, spread evenly, the embedding in front of the first and the
    head behind the last (the placement whose first and last stages are heavy under large vocabularies, paper Section 2.2)."""
    import torch
    if not 1 <= n_stages <= layers:
        raise ValueError("at least one layer for every stage")
    dtype = torch.bfloat16 if dtype is None else dtype
    g = torch.Generator(device=device).manual_seed(seed)
    stages = []
    for s in range(n_stages):
        of_stage = [Embedding(vocab, width, dtype, device, g)] if s == 0 else []
        for _ in range(layers * s // n_stages, layers * (s + 1) // n_stages):
            of_stage += [Recurrence(width, dtype, device, g), FeedForward(width, hidden, dtype, device=device, generator=g)]
        stages.append(Stage(of_stage + ([Head(vocab, width, dtype, device=device, generator=g)] if s == n_stages - 1 else [])))
    return stages
