"""What the stage operators refuse, without a GPU: the C ABI returns before it looks at a pointer, and the Python functions check tensors."""
import ctypes
import os
import re

import pytest
import torch

import paper_2510_05112_amd as fp
from paper_2510_05112_amd import stage_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ENOMEM, ENODEV, OK = -1, -2, -5, 0
P = 1 << 20   # a pointer that nothing looks at


@pytest.fixture(scope="module")
def lib():
    return ops._lib()


def test_library_exports_every_declared_operator(lib):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "fpsched_ops.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(fpsched_op_[a-z_]+)\s*\(", header))
    assert len(names) == 13
    for n in names:
        assert hasattr(lib, n), n


def called(f, defaults, **changes):
    return f(*dict(defaults, **changes).values())


EMBEDDING = dict(device=-1, type=0, table=P, table_stride=64, rows=10, width=64, tokens=P, wide=0, n=5, scale=1.0, out=P, out_stride=64, stream=None)
EMBEDDING_GRAD = dict(device=-1, type=0, grad=P, grad_stride=64, rows=10, width=64, tokens=P, wide=0, n=5, scale=1.0, out_type=2, out=P, out_stride=64, accumulate=0,
                      workspace=P, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(type=3), dict(type=-1), dict(rows=-1), dict(width=-1), dict(n=-1), dict(table_stride=63), dict(out_stride=63), dict(width=1 << 21, table_stride=1 << 22, out_stride=1 << 22)])
def test_embedding(lib, change):
    assert called(lib.fpsched_op_embedding, EMBEDDING) == ENODEV
    assert called(lib.fpsched_op_embedding, EMBEDDING, **change) == EINVAL


@pytest.mark.parametrize("change", [dict(type=3), dict(out_type=1), dict(out_type=0, accumulate=1), dict(rows=-1), dict(n=1 << 31), dict(rows=1 << 31), dict(grad_stride=60),
                                    dict(out_stride=60)])
def test_embedding_grad(lib, change):
    assert called(lib.fpsched_op_embedding_grad, EMBEDDING_GRAD) == ENODEV
    assert called(lib.fpsched_op_embedding_grad, EMBEDDING_GRAD, **change) == EINVAL


@pytest.mark.parametrize("change", [dict(workspace=None), dict(workspace=P + 8), dict(out=None), dict(grad=None), dict(tokens=None)])
def test_embedding_grad_pointers(lib, change):
    assert called(lib.fpsched_op_embedding_grad, dict(EMBEDDING_GRAD, device=0), **change) == EINVAL
    assert called(lib.fpsched_op_embedding_grad, dict(EMBEDDING_GRAD, device=0), bytes=100) == ENOMEM


def strides(*values):
    return (ctypes.c_int64 * len(values))(*values)


RECURRENCE = dict(device=-1, type=0, batch=4, steps=5000, width=66, gate=P, value=P, strides=strides(*[330000, 66] * 3), state=None, lengths=None, out=P, final=P, kept=None,
                  workspace=P, bytes=1 << 30, stream=None)
RECURRENCE_GRAD = dict(device=-1, type=0, batch=4, steps=5000, width=66, grad=P, gate=P, value=P, strides=strides(*[330000, 66] * 5), kept=P, grad_state=None, lengths=None,
                       d_gate=P, d_value=P, d_state=P, workspace=P, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change", [dict(type=3), dict(batch=-1), dict(batch=1 << 16), dict(steps=-1), dict(width=-1), dict(width=(1 << 24) + 1), dict(strides=None),
                                    dict(strides=strides(330000, -66, 330000, 66, 330000, 66)), dict(strides=strides(330000, 66, 330000, 66, 330000, 65)),
                                    dict(strides=strides(330000, 66, 330000, 66, 0, 66)), dict(strides=strides(1 << 32, 66, 330000, 66, 330000, 66))])
def test_recurrence(lib, change):
    assert called(lib.fpsched_op_recurrence, RECURRENCE) == ENODEV
    assert called(lib.fpsched_op_recurrence, RECURRENCE, **change) == EINVAL


def test_recurrence_pointers_and_workspace(lib):
    on = dict(RECURRENCE, device=0)
    for change in (dict(gate=None), dict(out=None), dict(final=None), dict(workspace=None), dict(workspace=P + 4)):
        assert called(lib.fpsched_op_recurrence, on, **change) == EINVAL
    assert called(lib.fpsched_op_recurrence, on, bytes=64) == ENOMEM
    assert called(lib.fpsched_op_recurrence, on, batch=0) == OK
    on = dict(RECURRENCE_GRAD, device=0)
    for change in (dict(kept=None), dict(d_gate=None), dict(grad=None), dict(workspace=None), dict(strides=strides(*[330000, 66] * 4, 330000, 0))):
        assert called(lib.fpsched_op_recurrence_grad, on, **change) == EINVAL
    assert called(lib.fpsched_op_recurrence_grad, on, bytes=64) == ENOMEM


FFN = dict(device=-1, type=0, act=0, tokens=20, width=64, hidden=128, x=P, x_stride=64, w_in=P, w_out=P, kept=P, h=P, out=P, out_stride=64, workspace=P, bytes=1 << 30, stream=None)
FFN_B = dict(device=-1, type=0, act=0, tokens=20, width=64, hidden=128, grad=P, grad_stride=64, w_in=P, w_out=P, kept=P, d_x=P, d_x_stride=64, workspace=P,
             bytes=1 << 30, stream=None)
FFN_W = dict(device=-1, type=0, tokens=20, width=64, hidden=128, x=P, x_stride=64, grad=P, grad_stride=64, kept=P, out_type=2, d_w_in=P, d_w_out=P, accumulate=0,
             workspace=P, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("name,defaults", [("ffn", FFN), ("ffn_input_grad", FFN_B), ("ffn_weight_grad", FFN_W)])
def test_ffn(lib, name, defaults):
    f = getattr(lib, "fpsched_op_" + name)
    assert called(f, defaults) == ENODEV
    changes = [dict(type=2), dict(tokens=-1), dict(width=60), dict(hidden=0), dict(hidden=132), dict(width=(1 << 21) + 8)]
    changes += [dict(act=3), dict(act=-1)] if "act" in defaults else [dict(out_type=1), dict(out_type=0, accumulate=1)]
    changes += [{key: 56} for key in defaults if key.endswith("stride")]
    for change in changes:
        assert called(f, defaults, **change) == EINVAL, change
    on = dict(defaults, device=0)
    pointers = [key for key in defaults if defaults[key] == P and key != "workspace" and not (key == "kept" and name == "ffn")]
    for change in [{key: bad} for key in pointers for bad in (None, P + 8)] + [{key: 68} for key in defaults if key.endswith("stride")]:
        assert called(f, on, **change) == EINVAL, change


LOGPROBS = dict(device=-1, type=0, rows=9, vocab=50000, logits=P, stride=50000, tokens=P, wide=0, k=8, logprob=P, entropy=P, lse=P, ids=P, alternatives=P, workspace=P,
                bytes=1 << 30, stream=None)
LOGPROBS_GRAD = dict(device=-1, type=0, rows=9, vocab=50000, logits=P, stride=50000, tokens=P, wide=0, lse=P, entropy=P, gl=None, ge=None, out=P, out_stride=50000, stream=None)


@pytest.mark.parametrize("change", [dict(type=4), dict(rows=-1), dict(vocab=0), dict(stride=49999), dict(k=33), dict(k=-1), dict(rows=1 << 31), dict(vocab=1 << 31, stride=1 << 31)])
def test_logprobs(lib, change):
    assert called(lib.fpsched_op_logprobs, LOGPROBS) == ENODEV
    assert called(lib.fpsched_op_logprobs, LOGPROBS, **change) == EINVAL


def test_logprobs_pointers_and_workspace(lib):
    on = dict(LOGPROBS, device=0)
    for change in (dict(logits=None), dict(logits=P + 1), dict(tokens=None), dict(lse=None), dict(ids=None), dict(workspace=None), dict(workspace=P + 8)):
        assert called(lib.fpsched_op_logprobs, on, **change) == EINVAL, change
    assert called(lib.fpsched_op_logprobs, on, bytes=64) == ENOMEM
    assert called(lib.fpsched_op_logprobs_grad, LOGPROBS_GRAD) == ENODEV
    for change in (dict(out_stride=49999), dict(stride=1), dict(type=3), dict(vocab=0)):
        assert called(lib.fpsched_op_logprobs_grad, LOGPROBS_GRAD, **change) == EINVAL, change
    for change in (dict(stride=50008), dict(out=P + 1), dict(logits=P + 3), dict(lse=None), dict(out=None)):   # (the first: in place, with another stride)
        assert called(lib.fpsched_op_logprobs_grad, dict(LOGPROBS_GRAD, device=0), **change) == EINVAL, change


def test_python_functions_need_cuda_tensors():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(128, 64, dtype=torch.bfloat16)
    tokens = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ops.embedding(w, tokens), lambda: ops.embedding_grad(x, tokens, 5), lambda: ops.gated_recurrence(x[None], x[None]),
                 lambda: ops.gated_recurrence_grad(x[None], x[None], x[None], x[None]), lambda: ops.gated_ffn(x, w, w.t()),
                 lambda: ops.gated_ffn_input_grad(x, w, w.t(), {}), lambda: ops.gated_ffn_weight_grad(x, x, {}, {}), lambda: ops.token_logprobs(x, tokens),
                 lambda: ops.token_logprobs_grad(x, tokens, x, x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


@pytest.mark.gpu
def test_python_functions_check_their_tensors():
    def zeros(*shape, dtype=torch.bfloat16):
        return torch.zeros(shape, dtype=dtype, device="cuda")
    x, w_in, w_out, tokens = zeros(4, 64), zeros(64, 64), zeros(64, 32), zeros(4, dtype=torch.int32)
    f = torch.float32
    for call in (lambda: ops.embedding(w_in, tokens.float()), lambda: ops.embedding(w_in.t(), tokens), lambda: ops.embedding(w_in.double(), tokens),
                 lambda: ops.embedding(w_in, tokens, out=zeros(4, 64, dtype=f)), lambda: ops.embedding(w_in, tokens.cpu()),
                 lambda: ops.embedding_grad(x, tokens[:3], 9), lambda: ops.embedding_grad(x, tokens, 9, accumulate=True), lambda: ops.embedding_grad(x, tokens, -1),
                 lambda: ops.embedding_grad(x, tokens, 9, out=zeros(9, 64), accumulate=True), lambda: ops.embedding_grad(x, tokens, 9, out=zeros(8, 64)),
                 lambda: ops.gated_recurrence(x, x), lambda: ops.gated_recurrence(x[None], x[None].float()), lambda: ops.gated_recurrence(x[None], x[None], zeros(1, 64)),
                 lambda: ops.gated_recurrence(x[None], x[None], lengths=zeros(1, dtype=torch.int64)), lambda: ops.gated_recurrence(x.t()[None], x.t()[None]),
                 lambda: ops.gated_recurrence_grad(x[None], x[None], x[None], zeros(1, 2, 64, dtype=f)),
                 lambda: ops.gated_ffn(x, w_in, w_out, "tanh"), lambda: ops.gated_ffn(x.float(), w_in.float(), w_out.float()), lambda: ops.gated_ffn(x, w_in, w_out.t()),
                 lambda: ops.gated_ffn(x, w_in[:63], w_out), lambda: ops.gated_ffn(zeros(4, 65)[:, 1:], w_in, w_out), lambda: ops.gated_ffn(x[:, :60], w_in[:, :60].contiguous(), w_out[:60]),
                 lambda: ops.gated_ffn_input_grad(x, w_in, w_out, dict(pre=zeros(4, 60), hidden=zeros(4, 30))), lambda: ops.gated_ffn_input_grad(x, w_in, w_out, dict(pre=zeros(4, 64), hidden=zeros(4, 32))),
                 lambda: ops.gated_ffn_weight_grad(x, x, dict(pre=zeros(4, 64), hidden=zeros(4, 32)), dict(pre=zeros(4, 64), hidden=zeros(4, 32))),
                 lambda: ops.token_logprobs(x, tokens, 33), lambda: ops.token_logprobs(x, tokens[:2]), lambda: ops.token_logprobs(x[0], tokens),
                 lambda: ops.token_logprobs_grad(x, tokens, zeros(4, dtype=f), zeros(4, dtype=f)),
                 lambda: ops.token_logprobs(x, tokens, workspace=torch.zeros(100, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fp.FpschedError):   # (rows in one place)
        ops.token_logprobs(zeros(1, 64).expand(4, 64), tokens)
    with pytest.raises(fp.FpschedError):
        ops.embedding_grad(x, tokens, 9, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))


def test_more_tokens_than_a_gradient_has_room_for(lib):
    assert called(lib.fpsched_op_embedding_grad, EMBEDDING_GRAD, n=1 << 30) == EINVAL
    assert lib.fpsched_op_embedding_grad_workspace_bytes(10, 64, 1 << 30) == 0
    assert lib.fpsched_op_embedding_grad_workspace_bytes(10, 64, (1 << 30) - 1) > 0


@pytest.mark.parametrize("name,defaults,changes", [
    ("embedding", EMBEDDING, [dict(table=P + 1), dict(out=P + 1), dict(type=2, out=P + 2)]),
    ("embedding_grad", EMBEDDING_GRAD, [dict(grad=P + 1), dict(out=P + 2)]),
    ("recurrence", RECURRENCE, [dict(gate=P + 1), dict(value=P + 1), dict(out=P + 1), dict(type=2, out=P + 2)]),
    ("recurrence_grad", RECURRENCE_GRAD, [dict(grad=P + 1), dict(gate=P + 1), dict(value=P + 1), dict(d_gate=P + 1), dict(d_value=P + 1)])])
def test_tensors_that_are_not_aligned_to_their_elements(lib, name, defaults, changes):
    for change in changes:
        assert called(getattr(lib, "fpsched_op_" + name), dict(defaults, device=0), **change) == EINVAL, change
