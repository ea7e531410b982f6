"""Operators that the items of a language model's pipeline stages run, on the GPU (C ABI: include/fpsched_ops.h).

A schedule orders items, and the cost table of a ``Problem`` says what each costs; these are what the items of a model's stages compute,
split the way the items are split:

    first stage    ``embedding`` (F), ``embedding_grad`` (W)
    inner stages   ``gated_recurrence`` (F), ``gated_recurrence_grad`` (B)
                   ``gated_ffn`` (F), ``gated_ffn_input_grad`` (B), ``gated_ffn_weight_grad`` (W)
    last stage     ``token_logprobs`` (F), ``token_logprobs_grad`` (B)

``tuner.measure_costs`` times stages made of them.  As elsewhere in the package the functions only check and marshal arguments: CUDA
tensors in, CUDA tensors out, asynchronous on ``stream`` (default: the device's current one), on the GPU the tensors are on
whether or not that is the current one.  What is not handed in (``out``, ``workspace``) is allocated on that stream.  The
gradients are calls of their own; autograd takes no part: an output never requires a gradient, also where an input does.  Wrong arguments raise ``ValueError``, what the library refuses ``FpschedError``.
"""
from __future__ import annotations

import ctypes

from .binding import FpschedError, load_library

BLOCK = 64   # steps between the states that ``gated_recurrence`` keeps (FPSCHED_RECURRENCE_BLOCK)
MAX_ALTERNATIVES = 32
_ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}

_declared = None


def _lib():
    global _declared
    if _declared is None:
        lib = load_library()
        vp, i32, i64, f32, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        ws = [vp, size, vp]   # workspace, its bytes, stream
        calls = {
            "embedding": [i32, i32, vp, i64, i64, i64, vp, i32, i64, f32, vp, i64, vp],
            "embedding_grad": [i32, i32, vp, i64, i64, i64, vp, i32, i64, f32, i32, vp, i64, i32] + ws,
            "recurrence": [i32, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp] + ws,
            "recurrence_grad": [i32, i32, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp] + ws,
            "ffn": [i32, i32, i32, i64, i64, i64, vp, i64, vp, vp, vp, vp, vp, i64] + ws,
            "ffn_input_grad": [i32, i32, i32, i64, i64, i64, vp, i64, vp, vp, vp, vp, i64] + ws,
            "ffn_weight_grad": [i32, i32, i64, i64, i64, vp, i64, vp, i64, vp, i32, vp, vp, i32] + ws,
            "logprobs": [i32, i32, i64, i64, vp, i64, vp, i32, i32, vp, vp, vp, vp, vp] + ws,
            "logprobs_grad": [i32, i32, i64, i64, vp, i64, vp, i32, vp, vp, vp, vp, vp, i64, vp],
        }
        for name, args in calls.items():
            f = getattr(lib, "fpsched_op_" + name)
            f.restype, f.argtypes = ctypes.c_int, args
        for name, n in (("embedding_grad", 3), ("recurrence", 3), ("ffn", 3)):
            f = getattr(lib, f"fpsched_op_{name}_workspace_bytes")
            f.restype, f.argtypes = size, [i64] * n
        lib.fpsched_op_logprobs_workspace_bytes.restype = size
        lib.fpsched_op_logprobs_workspace_bytes.argtypes = [i64, i64, i32]
        _declared = lib
    return _declared


# ---- arguments -------------------------------------------------------------------------------------------------------
# (messages are put together only where they are raised: a call's checks take as long as its launch otherwise)

torch = None   # (imported by the first call: the package loads without it)
_TYPES = _HALVES = _INTS = _FLOAT = _INT = None


def _import():
    global torch, _TYPES, _HALVES, _INTS, _FLOAT, _INT
    import torch as module
    _TYPES = {module.bfloat16: 0, module.float16: 1, module.float32: 2}
    _HALVES = (module.bfloat16, module.float16)
    _INTS, _FLOAT, _INT = (module.int32, module.int64), (module.float32,), (module.int32,)
    torch = module


def _tensor(t, name, device, shape=None, dtypes=None, rows=False):
    """Checks a CUDA tensor; rows: the last dimension adjacent, else contiguous."""
    if not isinstance(t, torch.Tensor) or t.device != device:
        raise ValueError(f"{name}: a tensor on {device} is needed")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{name}: type {t.dtype}, expected one of {tuple(dtypes)}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous() and not (rows and (t.shape[-1] <= 1 or t.stride(-1) == 1)):
        raise ValueError(f"{name}: the elements of its last dimension have to be adjacent" if rows else f"{name}: has to be contiguous")
    return t


def _device(t, name):
    if torch is None:
        _import()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name}: a CUDA tensor is needed")
    return t.device


def _matrix_stride(t):
    """Elements between the rows of a matrix (of one row: its width)."""
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _tokens(t, name, device, shape=None):
    _tensor(t, name, device, shape, _INTS)
    return int(t.dtype == torch.int64)


class _Stream:
    """The stream of a call; one that is handed in is current while the call's tensors are allocated, so that their memory belongs to it."""

    def __init__(self, stream, device):
        self.device, self.context = device, None
        if stream is None:
            self.stream = torch.cuda.current_stream(device.index)
        else:
            if stream.device != device:
                raise ValueError(f"the stream is one of {stream.device}, the tensors are on {device}")
            self.stream, self.context = stream, torch.cuda.stream(stream)

    def __enter__(self):
        if self.context is not None:
            self.context.__enter__()
        return self

    def __exit__(self, *exc):
        return self.context.__exit__(*exc) if self.context is not None else None

    def empty(self, *shape, dtype):
        return torch.empty(shape, dtype=dtype, device=self.device)

    def room(self, workspace, nbytes):
        """Place and size of the call's workspace (16 bytes or fewer: none is looked at)."""
        if workspace is not None:
            _tensor(workspace, "workspace", self.device)
        elif nbytes <= 16:
            return None, 0
        else:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.kept = workspace
        return workspace.data_ptr(), workspace.numel() * workspace.element_size()

    def call(self, name, *args):
        rc = getattr(_lib(), "fpsched_op_" + name)(self.device.index, *args, self.stream.cuda_stream)
        if rc != 0:
            raise FpschedError(rc, "fpsched_op_" + name)


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- embedding -------------------------------------------------------------------------------------------------------

def embedding(table, tokens, scale: float = 1.0, out=None, stream=None):
    """scale * table[tokens], with zeros for tokens outside the table (-1 for padding).  table: [rows][width], rows any distance
    apart; tokens: int32 or int64, any shape.  Returns [*tokens.shape][width] of the table's type."""
    device = _device(table, "table")
    if table.dim() != 2:
        raise ValueError("table: two dimensions are needed")
    _tensor(table, "table", device, dtypes=_TYPES, rows=True)
    wide = _tokens(tokens, "tokens", device)
    with _Stream(stream, device) as s:
        shape = (*tokens.shape, table.shape[1])
        if out is None:
            out = s.empty(*shape, dtype=table.dtype)
        else:
            _tensor(out, "out", device, shape, (table.dtype,))
        s.call("embedding", _TYPES[table.dtype], table.data_ptr(), _matrix_stride(table), table.shape[0], table.shape[1],
               tokens.data_ptr(), wide, tokens.numel(), float(scale), out.data_ptr(), table.shape[1])
    return out


def embedding_grad(grad, tokens, rows: int, scale: float = 1.0, out=None, accumulate: bool = False, workspace=None, stream=None):
    """The gradient of an embedding table of ``rows`` rows: every row's sum of the gradients of its tokens, times scale.  grad:
    [n][width] with rows any distance apart, or [*tokens.shape][width] contiguous; out: [rows][width] of grad's type (the default) or
    float32; accumulate: added to a float32 ``out`` (micro-batch by micro-batch) instead of written.  The same bits every time."""
    device = _device(grad, "grad")
    wide = _tokens(tokens, "tokens", device)
    rows = int(rows)
    if rows < 0:
        raise ValueError("rows: not negative")
    if grad.dim() < 1 or grad.shape[:-1] != tokens.shape:
        raise ValueError("grad: one row for every token")
    _tensor(grad, "grad", device, dtypes=_TYPES, rows=grad.dim() == 2)
    width = grad.shape[-1]
    flat = grad if grad.dim() == 2 else grad.view(tokens.numel(), width)
    if accumulate and (out is None or out.dtype != torch.float32):
        raise ValueError("accumulate: needs a float32 out")
    with _Stream(stream, device) as s:
        if out is None:
            out = s.empty(rows, width, dtype=grad.dtype)
        else:
            _tensor(out, "out", device, (rows, width), (grad.dtype, torch.float32), rows=True)
        room = s.room(workspace, _lib().fpsched_op_embedding_grad_workspace_bytes(rows, width, tokens.numel()))
        s.call("embedding_grad", _TYPES[grad.dtype], flat.data_ptr(), _matrix_stride(flat), rows, width, tokens.data_ptr(), wide,
               tokens.numel(), float(scale), _TYPES[out.dtype], out.data_ptr(), _matrix_stride(out), int(accumulate), *room)
    return out


# ---- gated linear recurrence -----------------------------------------------------------------------------------------

def _steps(*tensors):
    """HOST array of the sequence and step strides of [batch][steps][width] tensors (0 where there is one of them only)."""
    found = []
    for t in tensors:
        found += [t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0]
    return (ctypes.c_int64 * len(found))(*found)


def gated_recurrence(gate, value, state=None, lengths=None, keep: bool = False, out=None, final_state=None, workspace=None, stream=None):
    """h[t] = a[t] h[t-1] + (1 - a[t]) value[t] with a = sigmoid(gate), per sequence and channel.  gate, value: [batch][steps][width],
    channels adjacent; state: float32 [batch][width] in front of the first step (default: zero); lengths: int32 [batch], the steps of each
    sequence (behind them the output is zero and the state stands still).  Returns dict(out, state: float32 [batch][width] behind
    the last step, kept: with ``keep``, what ``gated_recurrence_grad`` needs).  ``final_state`` may be ``state`` itself: a serving
    loop calls this with one step at a time."""
    device = _device(value, "value")
    if value.dim() != 3:
        raise ValueError("value: [batch][steps][width]")
    n, steps, width = value.shape
    _tensor(value, "value", device, dtypes=_TYPES, rows=True)
    _tensor(gate, "gate", device, (n, steps, width), (value.dtype,), rows=True)
    for name, t in (("state", state), ("final_state", final_state)):
        if t is not None:
            _tensor(t, name, device, (n, width), _FLOAT)
    if lengths is not None:
        _tensor(lengths, "lengths", device, (n,), _INT)
    with _Stream(stream, device) as s:
        if out is None:
            out = s.empty(n, steps, width, dtype=value.dtype)
        else:
            _tensor(out, "out", device, (n, steps, width), (value.dtype,), rows=True)
        if final_state is None:
            final_state = s.empty(n, width, dtype=torch.float32)
        kept = s.empty(n, -(-steps // BLOCK), width, dtype=torch.float32) if keep else None
        room = s.room(workspace, _lib().fpsched_op_recurrence_workspace_bytes(n, steps, width))
        s.call("recurrence", _TYPES[value.dtype], n, steps, width, gate.data_ptr(), value.data_ptr(), _steps(gate, value, out), _ptr(state),
               _ptr(lengths), out.data_ptr(), final_state.data_ptr(), _ptr(kept), *room)
    return dict(out=out, state=final_state, **({"kept": kept} if keep else {}))


def gated_recurrence_grad(grad, gate, value, kept, grad_state=None, lengths=None, workspace=None, stream=None):
    """Gradients of ``gated_recurrence`` (called with ``keep`` on the same gate, value, state and lengths): grad is that of its output,
    grad_state (float32 [batch][width], default: zero) that of its final state.  Returns dict(gate, value, state)."""
    device = _device(value, "value")
    if value.dim() != 3:
        raise ValueError("value: [batch][steps][width]")
    n, steps, width = value.shape
    _tensor(value, "value", device, dtypes=_TYPES, rows=True)
    for name, t in (("gate", gate), ("grad", grad)):
        _tensor(t, name, device, (n, steps, width), (value.dtype,), rows=True)
    _tensor(kept, "kept", device, (n, -(-steps // BLOCK), width), _FLOAT)
    if grad_state is not None:
        _tensor(grad_state, "grad_state", device, (n, width), _FLOAT)
    if lengths is not None:
        _tensor(lengths, "lengths", device, (n,), _INT)
    with _Stream(stream, device) as s:
        d_gate, d_value = (s.empty(n, steps, width, dtype=value.dtype) for _ in range(2))
        d_state = s.empty(n, width, dtype=torch.float32)
        room = s.room(workspace, _lib().fpsched_op_recurrence_workspace_bytes(n, steps, width))
        s.call("recurrence_grad", _TYPES[value.dtype], n, steps, width, grad.data_ptr(), gate.data_ptr(), value.data_ptr(),
               _steps(grad, gate, value, d_gate, d_value), kept.data_ptr(), _ptr(grad_state), _ptr(lengths), d_gate.data_ptr(),
               d_value.data_ptr(), d_state.data_ptr(), *room)
    return dict(gate=d_gate, value=d_value, state=d_state)


# ---- gated feed-forward block ----------------------------------------------------------------------------------------

def _ffn_sizes(x, name, w_in, w_out, device):
    if x.dim() != 2:
        raise ValueError(f"{name}: [tokens][width]")
    tokens, width = x.shape
    _tensor(x, name, device, dtypes=_HALVES, rows=True)
    if w_in.dim() != 2 or w_in.shape[0] % 2:
        raise ValueError("w_in: [2 hidden][width]")
    hidden = w_in.shape[0] // 2
    _tensor(w_in, "w_in", device, (2 * hidden, width), (x.dtype,))
    _tensor(w_out, "w_out", device, (width, hidden), (x.dtype,))
    _multiples_of_8(width, hidden)
    return tokens, width, hidden


def _multiples_of_8(width, hidden):
    if width <= 0 or hidden <= 0 or width % 8 or hidden % 8:
        raise ValueError("width and hidden width: multiples of 8")


def _rows_of_16_bytes(**tensors):
    for name, t in tensors.items():
        if t.data_ptr() % 16 or _matrix_stride(t) % 8:
            raise ValueError(f"{name}: its rows have to begin at multiples of 16 bytes")


def _activation(name):
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation: one of {sorted(_ACTIVATIONS)}")
    return _ACTIVATIONS[name]


def _kept_views(room, tokens, hidden, dtype):
    """The memory that a feed-forward block keeps, as the B item leaves it: d_pre and hidden."""
    both = room.view(dtype)
    n = 2 * tokens * hidden
    pre = both[:n].view(tokens, 2 * hidden)
    pre.numbers_of = "F"   # (the item whose numbers are in that memory: copies of the dict share the tensor)
    return dict(pre=pre, hidden=both[n:].view(tokens, hidden))


def _kept_memory(kept, tokens, hidden, dtype, device):
    pre, h = kept["pre"], kept["hidden"]
    _tensor(pre, "kept", device, (tokens, 2 * hidden), (dtype,))
    _tensor(h, "kept", device, (tokens, hidden), (dtype,))
    if h.untyped_storage().data_ptr() != pre.untyped_storage().data_ptr() or h.data_ptr() != pre.data_ptr() + 4 * tokens * hidden:
        raise ValueError("kept: not the memory that gated_ffn returned")
    return pre


def _kept_item(memory):
    """Whose numbers are kept.  (Views that a caller has made do not say.)"""
    return getattr(memory, "numbers_of", None)


def gated_ffn(x, w_in, w_out, activation: str = "silu", keep: bool = False, out=None, workspace=None, stream=None):
    """(act(x w_gate^T) * (x w_up^T)) w_out^T, with w_in = [w_gate; w_up].  x: [tokens][width], rows any distance apart; w_in: [2
    hidden][width]; w_out: [width][hidden]; bfloat16 or float16; widths multiples of 8.  Between the products hidden is rounded to that
    type, and so is what ``gated_ffn_input_grad`` multiplies by w_in.  Returns dict(out, kept: with ``keep``, what the two gradients
    need, six bytes for each token and hidden channel)."""
    device = _device(x, "x")
    tokens, width, hidden = _ffn_sizes(x, "x", w_in, w_out, device)
    act = _activation(activation)
    with _Stream(stream, device) as s:
        if out is None:
            out = s.empty(tokens, width, dtype=x.dtype)
        else:
            _tensor(out, "out", device, (tokens, width), (x.dtype,), rows=True)
        _rows_of_16_bytes(x=x, w_in=w_in, w_out=w_out, out=out)
        kept = s.empty(6 * tokens * hidden, dtype=torch.uint8) if keep else None
        h = s.empty(tokens, hidden, dtype=x.dtype)
        room = s.room(workspace, _lib().fpsched_op_ffn_workspace_bytes(tokens, width, hidden))
        s.call("ffn", _TYPES[x.dtype], act, tokens, width, hidden, x.data_ptr(), _matrix_stride(x), w_in.data_ptr(), w_out.data_ptr(), _ptr(kept),
               h.data_ptr(), out.data_ptr(), _matrix_stride(out), *room)
    return dict(out=out, **({"kept": _kept_views(kept, tokens, hidden, x.dtype)} if keep else {}))


def gated_ffn_input_grad(grad, w_in, w_out, kept, activation: str = "silu", workspace=None, stream=None):
    """The B item: the gradient of x from that of the output and what ``gated_ffn`` kept.  Returns dict(x, kept: what
    ``gated_ffn_weight_grad`` needs).  It takes the place of what was kept: this is called once for each ``gated_ffn`` (ValueError)."""
    device = _device(grad, "grad")
    tokens, width, hidden = _ffn_sizes(grad, "grad", w_in, w_out, device)
    act = _activation(activation)
    memory = _kept_memory(kept, tokens, hidden, grad.dtype, device)
    if _kept_item(memory) == "B":
        raise ValueError("kept: gated_ffn_input_grad has taken its place, once for each gated_ffn")
    _rows_of_16_bytes(grad=grad, w_in=w_in, w_out=w_out, kept=memory)
    with _Stream(stream, device) as s:
        d_x = s.empty(tokens, width, dtype=grad.dtype)
        room = s.room(workspace, _lib().fpsched_op_ffn_workspace_bytes(tokens, width, hidden))
        s.call("ffn_input_grad", _TYPES[grad.dtype], act, tokens, width, hidden, grad.data_ptr(), _matrix_stride(grad), w_in.data_ptr(),
               w_out.data_ptr(), memory.data_ptr(), d_x.data_ptr(), width, *room)
    memory.numbers_of = "B"
    return dict(x=d_x, kept=dict(pre=kept["pre"], hidden=kept["hidden"]))


def gated_ffn_weight_grad(x, grad, kept, grad_kept, out=None, accumulate: bool = False, workspace=None, stream=None):
    """The W item: the weights' gradients from x, the output's gradient, what ``gated_ffn`` kept and what ``gated_ffn_input_grad``
    made of it.  out: dict(w_in, w_out) of tensors of x's type or, both, float32; accumulate: added to float32 ones.  Returns them."""
    device = _device(x, "x")
    if x.dim() != 2:
        raise ValueError("x: [tokens][width]")
    tokens, width = x.shape
    _tensor(x, "x", device, dtypes=_HALVES, rows=True)
    _tensor(grad, "grad", device, (tokens, width), (x.dtype,), rows=True)
    hidden = kept["hidden"].shape[-1]
    _multiples_of_8(width, hidden)
    memory = _kept_memory(grad_kept, tokens, hidden, x.dtype, device)
    if kept["pre"].data_ptr() != memory.data_ptr():
        raise ValueError("grad_kept: of another call than kept")
    if _kept_item(memory) == "F":
        raise ValueError("grad_kept: gated_ffn_input_grad comes first")
    if accumulate and (out is None or out["w_in"].dtype != torch.float32):
        raise ValueError("accumulate: needs float32 outputs")
    with _Stream(stream, device) as s:
        if out is None:
            out = dict(w_in=s.empty(2 * hidden, width, dtype=x.dtype), w_out=s.empty(width, hidden, dtype=x.dtype))
        kind = out["w_in"].dtype
        _tensor(out["w_in"], "out", device, (2 * hidden, width), (x.dtype, torch.float32))
        _tensor(out["w_out"], "out", device, (width, hidden), (kind,))
        _rows_of_16_bytes(x=x, grad=grad, kept=memory, w_in=out["w_in"], w_out=out["w_out"])
        room = s.room(workspace, _lib().fpsched_op_ffn_workspace_bytes(tokens, width, hidden))
        s.call("ffn_weight_grad", _TYPES[x.dtype], tokens, width, hidden, x.data_ptr(), _matrix_stride(x), grad.data_ptr(), _matrix_stride(grad),
               memory.data_ptr(), _TYPES[kind], out["w_in"].data_ptr(), out["w_out"].data_ptr(), int(accumulate), *room)
    return out


# ---- log probabilities -----------------------------------------------------------------------------------------------

def token_logprobs(logits, tokens, alternatives: int = 0, workspace=None, stream=None):
    """Log probabilities of given tokens.  logits: [rows][vocab], rows any distance apart; tokens: int32 or int64 [rows] (outside the
    vocabulary, -1 for padding: log probability 0).  Returns dict(logprob, entropy: float32 [rows], lse: float32 [rows][2], the log-sum-exp in
    two parts (largest logit, rest), and with ``alternatives`` = k > 0 the k largest logits of each row, of equal ones the
    lowest id first, as ids: int32 [rows][k] and logprobs: float32 [rows][k]; -1 and -inf where fewer are not masked).  A logit of
    -inf is masked; a row with nothing else has logprob -inf and entropy 0; one with NaN or +inf, padding or not, is NaN
    throughout (of lse, the rest)."""
    device = _device(logits, "logits")
    if logits.dim() != 2 or not logits.shape[1]:
        raise ValueError("logits: [rows][vocab]")
    n, vocab = logits.shape
    _tensor(logits, "logits", device, dtypes=_TYPES, rows=True)
    wide = _tokens(tokens, "tokens", device, (n,))
    k = int(alternatives)
    if not 0 <= k <= MAX_ALTERNATIVES:
        raise ValueError(f"alternatives: 0 to {MAX_ALTERNATIVES}")
    with _Stream(stream, device) as s:
        done = dict(logprob=s.empty(n, dtype=torch.float32), entropy=s.empty(n, dtype=torch.float32), lse=s.empty(n, 2, dtype=torch.float32))
        if k:
            done.update(ids=s.empty(n, k, dtype=torch.int32), logprobs=s.empty(n, k, dtype=torch.float32))
        room = s.room(workspace, _lib().fpsched_op_logprobs_workspace_bytes(n, vocab, k))
        s.call("logprobs", _TYPES[logits.dtype], n, vocab, logits.data_ptr(), _matrix_stride(logits), tokens.data_ptr(), wide, k,
               done["logprob"].data_ptr(), done["entropy"].data_ptr(), done["lse"].data_ptr(), _ptr(done.get("ids")), _ptr(done.get("logprobs")),
               *room)
    return done


def token_logprobs_grad(logits, tokens, lse, entropy, grad_logprob=None, grad_entropy=None, out=None, stream=None):
    """The gradient of the logits from those of ``logprob`` and ``entropy`` (float32 [rows], None: zero) and what ``token_logprobs``
    returned.  out: of the logits' type, may be ``logits`` itself.  Returns it."""
    device = _device(logits, "logits")
    if logits.dim() != 2 or not logits.shape[1]:
        raise ValueError("logits: [rows][vocab]")
    n, vocab = logits.shape
    _tensor(logits, "logits", device, dtypes=_TYPES, rows=True)
    wide = _tokens(tokens, "tokens", device, (n,))
    _tensor(lse, "lse", device, (n, 2), _FLOAT)
    _tensor(entropy, "entropy", device, (n,), _FLOAT)
    for name, t in (("grad_logprob", grad_logprob), ("grad_entropy", grad_entropy)):
        if t is not None:
            _tensor(t, name, device, (n,), _FLOAT)
    with _Stream(stream, device) as s:
        if out is None:
            out = s.empty(n, vocab, dtype=logits.dtype)
        else:
            _tensor(out, "out", device, (n, vocab), (logits.dtype,), rows=True)
        s.call("logprobs_grad", _TYPES[logits.dtype], n, vocab, logits.data_ptr(), _matrix_stride(logits), tokens.data_ptr(), wide, lse.data_ptr(),
               entropy.data_ptr(), _ptr(grad_logprob), _ptr(grad_entropy), out.data_ptr(), _matrix_stride(out))
    return out
