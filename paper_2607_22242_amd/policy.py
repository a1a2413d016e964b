"""ctypes binding of include/sched_policy.h, same names: the operators of an
agent that proposes mappings and learns from their makespans.

Argument marshalling only.  Tensors are torch tensors on one GPU; results are
new tensors unless they are given, and the calls enqueue their work on `stream`
(default: the current stream of the tensors' GPU) and return.  A tensor that
belongs to another stream is marked as used on this one; ordering the streams
is the caller's.  The calls take no part in automatic differentiation: results
of tensors that require a gradient do not, and each operator's gradient is a
call of its own (workloads/agent.py joins them to torch's).
"""
from __future__ import annotations

import ctypes
import math
import struct
from typing import Optional, Tuple

from . import binding as _b
from .binding import SchedError

POLICY_EXPORTED = ["sched_embed", "sched_embed_grad_workspace_bytes", "sched_embed_grad",
                   "sched_token_logprobs", "sched_token_logprobs_grad", "sched_group_advantages",
                   "sched_policy_loss", "sched_preference_loss",
                   "sched_attention_workspace_bytes", "sched_attention",
                   "sched_attention_grad_workspace_bytes", "sched_attention_grad",
                   "sched_shared_attention_workspace_bytes", "sched_shared_attention",
                   "sched_shared_attention_grad_workspace_bytes", "sched_shared_attention_grad",
                   "sched_norm_rotate", "sched_norm_rotate_grad_workspace_bytes",
                   "sched_norm_rotate_grad", "sched_beam_workspace_bytes", "sched_beam_select",
                   "sched_beam_reorder"]

_P, _I32, _I64, _F = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


class sched_matrix(ctypes.Structure):
    _fields_ = [("data", _P), ("dtype", _I32), ("rows", _I64), ("cols", _I64), ("stride", _I64)]


class sched_tokens(ctypes.Structure):
    _fields_ = [("data", _P), ("bits", _I32), ("n", _I64)]


class sched_policy_desc(ctypes.Structure):
    _fields_ = [("logits", sched_matrix), ("tokens", sched_tokens), ("old_logp", _P),
                ("ref_logp", _P), ("advantages", _P), ("weights", _P), ("clip_low", _F),
                ("clip_high", _F), ("kl_weight", _F), ("temperature", _F), ("loss_scale", _F),
                ("loss", _P), ("losses", _P), ("logp", _P), ("d_logits", sched_matrix)]


class sched_heads(ctypes.Structure):
    _fields_ = [("data", _P), ("row_stride", _I64), ("head_stride", _I64)]


class sched_attention_desc(ctypes.Structure):
    _fields_ = [("q", sched_heads), ("k", sched_heads), ("v", sched_heads), ("out", sched_heads),
                ("lse", _P), ("dtype", _I32), ("head_dim", _I32), ("q_heads", _I32),
                ("kv_heads", _I32), ("q_rows", _I64), ("k_rows", _I64), ("q_offsets", _P),
                ("k_offsets", _P), ("k_lengths", _P), ("n_seqs", _I32), ("causal", _I32),
                ("scale", _F)]


class sched_shared_desc(ctypes.Structure):
    _fields_ = [("own", sched_attention_desc), ("prefix_k", sched_heads),
                ("prefix_v", sched_heads), ("prefix_rows", _I64), ("prefix_offsets", _P),
                ("prefix_lengths", _P), ("group_offsets", _P), ("n_groups", _I32)]


class sched_shared_grads(ctypes.Structure):
    _fields_ = [(n, sched_heads) for n in ("d_out", "d_q", "d_k", "d_v", "d_prefix_k",
                                           "d_prefix_v")]


class sched_norm_rotate_desc(ctypes.Structure):
    _fields_ = [("q", sched_heads), ("k", sched_heads), ("v", sched_heads),
                ("q_out", sched_heads), ("k_out", sched_heads), ("v_out", sched_heads),
                ("dtype", _I32), ("head_dim", _I32), ("q_heads", _I32), ("kv_heads", _I32),
                ("rows", _I64), ("out_rows", _I64), ("positions", sched_tokens),
                ("places", sched_tokens), ("q_weight", _P), ("k_weight", _P),
                ("frequencies", _P), ("turned", _I32), ("interleaved", _I32), ("norm", _I32),
                ("eps", _F)]


class sched_beam_desc(ctypes.Structure):
    _fields_ = [("logits", sched_matrix), ("scores", _P), ("last", sched_tokens),
                ("end_token", _I64), ("n_groups", _I32), ("beams", _I32), ("width", _I32),
                ("stay", _I32), ("temperature", _F), ("new_scores", _P), ("parents", _P),
                ("tokens", _P), ("token_bits", _I32)]


class sched_states(ctypes.Structure):
    _fields_ = [("data", _P), ("outer", _I64), ("slots", _I64), ("rows", _I64),
                ("row_bytes", _I64), ("outer_stride", _I64), ("slot_stride", _I64),
                ("row_stride", _I64)]


_ARGS = {
    "sched_embed": [_P, _P, _F, _P, _P],
    "sched_embed_grad_workspace_bytes": [_I64, _I64, _P],
    "sched_embed_grad": [_P, _P, _F, _I32, _P, _P, ctypes.c_size_t, _P],
    "sched_token_logprobs": [_P, _P, _F, _P, _P],
    "sched_token_logprobs_grad": [_P, _P, _F, _P, _P, _P, _P],
    "sched_group_advantages": [_P, _P, _P, _I32, _P, _I32, _P, _I32, _P, _P, _P, ctypes.c_size_t,
                               _P],
    "sched_policy_loss": [_P, _P],
    "sched_preference_loss": [_P, _P, _P, _P, _I32, _F, _F, _F, _P, _P, _P, _P],
    "sched_attention_workspace_bytes": [_P, _P],
    "sched_attention": [_P, _P, ctypes.c_size_t, _P],
    "sched_attention_grad_workspace_bytes": [_P, _P],
    "sched_attention_grad": [_P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P],
    "sched_shared_attention_workspace_bytes": [_P, _P],
    "sched_shared_attention": [_P, _P, ctypes.c_size_t, _P],
    "sched_shared_attention_grad_workspace_bytes": [_P, _P],
    "sched_shared_attention_grad": [_P, _P, _P, ctypes.c_size_t, _P],
    "sched_norm_rotate": [_P, _P],
    "sched_norm_rotate_grad_workspace_bytes": [_P, _P],
    "sched_norm_rotate_grad": [_P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P],
    "sched_beam_workspace_bytes": [_P, _P],
    "sched_beam_select": [_P, _P, ctypes.c_size_t, _P],
    "sched_beam_reorder": [_P, _P, _P, _I32, _P],
}

_NO_HEADS, _NOWHERE = (0, 0, 0), (0, 64, 0)  # tensors that are not there


def _packer(kind):
    """What makes a structure's bytes from its values, those of structures in it
    in their places: a fifth of the time of making them one by one, in calls
    whose time is the host's (26 values: 0.26 us, not 1.4)."""
    codes = {_P: "Q", _I32: "i", _I64: "q", _F: "f"}
    form, at = "=", 0

    def walk(kind, base):
        nonlocal form, at
        for name, of in kind._fields_:
            place = base + getattr(kind, name).offset
            if issubclass(of, ctypes.Structure):
                walk(of, place)
            else:
                form += "x" * (place - at) + codes[of]
                at = place + ctypes.sizeof(of)
    walk(kind, 0)
    return struct.Struct(form + "x" * (ctypes.sizeof(kind) - at)).pack


(_pack_heads, _pack_attention, _pack_shared, _pack_grads, _pack_rotate, _pack_beam,
 _pack_states) = map(_packer, (sched_heads, sched_attention_desc, sched_shared_desc, sched_shared_grads,
                               sched_norm_rotate_desc, sched_beam_desc, sched_states))
_F32 = _F16 = _BF16 = _INT32 = _INT64 = None  # torch's types, once it is loaded
_torch = _types = None
_call = {}  # the library's functions


def _load():
    global _torch, _types, _F32, _F16, _BF16, _INT32, _INT64
    import torch
    L = _b.lib()
    for name, args in _ARGS.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = ctypes.c_int, args
        _call[name] = fn
    _F32, _F16, _BF16 = torch.float32, torch.float16, torch.bfloat16
    _INT32, _INT64 = torch.int32, torch.int64
    _types = {_F32: 0, _F16: 1, _BF16: 2}
    _torch = torch


def _refuse(code: int, where: str):
    raise SchedError(code, where)


class _Call:
    """The tensors of one call: their GPU, its stream, and what they are.  A
    call of some microseconds is mostly what happens here, so it asks each
    tensor for as little as it needs."""

    __slots__ = ("where", "like", "index", "stream", "ptr", "other")

    def __init__(self, where: str, first, stream):
        if _torch is None:
            _load()
        self.where = where
        index = first.get_device() if isinstance(first, _torch.Tensor) else -1
        if index < 0 or not first.is_cuda:
            _refuse(-3, where + ": tensors are on a GPU")
        self.index, self.like, self.stream = index, first, stream
        current = _torch._C._cuda_getCurrentRawStream(index)
        self.ptr = current if stream is None else stream.cuda_stream
        # Tensors made here belong to the call's stream, inputs to any.
        self.other = self.ptr != current

    def use(self, t):
        if t.get_device() != self.index:
            _refuse(-3, self.where + ": tensors are on one GPU")
        if self.other:
            t.record_stream(self.stream)

    def new(self, shape, dtype):
        if not self.other:
            return self.like.new_empty(*shape, dtype=dtype)
        with _torch.cuda.stream(self.stream):
            return self.like.new_empty(*shape, dtype=dtype)

    def like_of(self, t):
        """A new tensor of t's shape and type."""
        if not self.other:
            return _torch.empty_like(t, memory_format=_torch.contiguous_format)
        with _torch.cuda.stream(self.stream):
            return _torch.empty_like(t, memory_format=_torch.contiguous_format)

    def matrix_values(self, t) -> Tuple:
        if self.other or t.get_device() != self.index:
            self.use(t)
        kind = _types.get(t.dtype)
        if kind is None:
            _refuse(-3, self.where + ": float32, float16 or bfloat16")
        if t.dim() != 2:
            _refuse(-2, self.where + ": a matrix has two dimensions")
        rows, cols = t.shape
        stride, step = t.stride()
        if step != 1 and cols > 1:
            _refuse(-3, self.where + ": the elements of a row are next to each other")
        stride = stride if rows > 1 else max(stride, cols)
        return t.data_ptr(), kind, rows, cols, stride

    def matrix(self, t) -> sched_matrix:
        return sched_matrix(*self.matrix_values(t))

    def token_values(self, t) -> Tuple:
        if self.other or t.get_device() != self.index:
            self.use(t)
        dtype = t.dtype
        bits = 64 if dtype is _INT64 else 32 if dtype is _INT32 else 0
        if not bits or not t.is_contiguous():
            _refuse(-3, self.where + ": tokens are contiguous int32 or int64")
        return t.data_ptr(), bits, t.numel()

    def tokens(self, t) -> sched_tokens:
        return sched_tokens(*self.token_values(t))

    def vector(self, t, dtype, n: Optional[int] = None) -> int:
        if self.other or t.get_device() != self.index:
            self.use(t)
        if t.dtype is not dtype or not t.is_contiguous():
            _refuse(-3, f"{self.where}: a contiguous tensor of {dtype}")
        if n is not None and t.numel() != n:
            _refuse(-2, f"{self.where}: {n} values, not {t.numel()}")
        return t.data_ptr()

    def floats(self, t, n: int):
        """A 32-bit result of n values: new, or the tensor that is given."""
        if t is None:
            return self.new((n,), _F32)
        self.vector(t, _F32, n)
        return t

    def workspace(self, given, nbytes: int):
        """(tensor, address, bytes): the caller's workspace, or a new one."""
        if given is not None:
            self.use(given)
            return given, given.data_ptr(), given.numel() * given.element_size()
        if nbytes == 0:
            return None, None, 0
        ws = self.new((nbytes,), _torch.uint8)
        at = ws.data_ptr()
        if at % 256:  # not from torch's own allocator
            ws = self.new((nbytes + 256,), _torch.uint8)
            at = (ws.data_ptr() + 255) // 256 * 256
        return ws, at, nbytes

    def packed(self, pack, values) -> bytes:
        try:
            return pack(*values)
        except (struct.error, OverflowError):
            _refuse(-3, self.where + ": a number that its type does not hold")

    def done(self, name: str, *args):
        if _torch._C._cuda_getDevice() == self.index:
            rc = _call[name](*args, self.ptr)
        else:
            with _torch.cuda.device(self.index):
                rc = _call[name](*args, self.ptr)
        if rc:
            _refuse(rc, self.where)

    def bytes(self, name: str, *args) -> int:
        need = ctypes.c_size_t()
        rc = _call[name](*args, ctypes.byref(need))
        if rc:
            _refuse(rc, self.where)
        return need.value


def sched_embed(table, tokens, scale: float = 1.0, out=None, stream=None):
    """scale * table[tokens], zeros where a token is outside the table; shape
    tokens.shape + (dim,)."""
    c = _Call("sched_embed", table, stream)
    m, t = c.matrix(table), c.tokens(tokens)
    if out is None:
        out = c.new((t.n, m.cols), table.dtype)
    o = c.matrix(out)
    c.done("sched_embed", ctypes.byref(m), ctypes.byref(t), scale, ctypes.byref(o))
    return out if tokens.dim() == 1 else out.view(*tokens.shape, m.cols)


def sched_embed_grad(d_rows, tokens, vocab: int, scale: float = 1.0, out=None,
                     accumulate: bool = False, workspace=None, stream=None):
    """Gradient of sched_embed by its table (vocab x dim, of d_rows' type, or
    as `out`); with accumulate it is added to `out`.  d_rows has a row per
    token."""
    c = _Call("sched_embed_grad", d_rows, stream)
    if d_rows.dim() != 2:
        try:
            d_rows = d_rows.view(tokens.numel(), d_rows.shape[-1])
        except RuntimeError:
            _refuse(-3 if d_rows.shape[:-1].numel() == tokens.numel() else -2,
                    c.where + ": d_rows is a matrix, or its rows lie at one distance")
    m, t = c.matrix(d_rows), c.tokens(tokens)
    if out is None:
        if accumulate:
            _refuse(-1, c.where + ": accumulate needs out")
        out = c.new((vocab, m.cols), d_rows.dtype)
    o = c.matrix(out)
    if o.rows != vocab:
        _refuse(-2, c.where + ": out has a row per token of the vocabulary")
    need = c.bytes("sched_embed_grad_workspace_bytes", t.n, m.cols)
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_embed_grad", ctypes.byref(m), ctypes.byref(t), scale, int(accumulate),
           ctypes.byref(o), at, nbytes)
    return out


def sched_token_logprobs(logits, tokens, temperature: float = 1.0, logp=None, stream=None):
    """Log-probabilities (float32) of the tokens, one per row of logits."""
    c = _Call("sched_token_logprobs", logits, stream)
    m, t = c.matrix(logits), c.tokens(tokens)
    logp = c.floats(logp, t.n)
    c.done("sched_token_logprobs", ctypes.byref(m), ctypes.byref(t), temperature, logp.data_ptr())
    return logp


def sched_token_logprobs_grad(logits, tokens, logp, d_logp, temperature: float = 1.0,
                              d_logits=None, stream=None):
    """Gradient by the logits of sched_token_logprobs' result `logp`; d_logits
    may be the logits themselves."""
    c = _Call("sched_token_logprobs_grad", logits, stream)
    m, t = c.matrix(logits), c.tokens(tokens)
    if d_logits is None:
        d_logits = c.new((m.rows, m.cols), logits.dtype)
    d = c.matrix(d_logits)
    c.done("sched_token_logprobs_grad", ctypes.byref(m), ctypes.byref(t), temperature,
           c.vector(logp, _F32, t.n), c.vector(d_logp, _F32, t.n), ctypes.byref(d))
    return d_logits


_MEANS = {"tokens": 0, "sequences": 1}


def sched_group_advantages(makespans, limits, group_offsets, offsets, tokens, mean: str = "tokens",
                           advantages=None, weights=None, workspace=None, stream=None):
    """(advantages, weights) per token from the int64 makespans of answers:
    answers group_offsets[g]..group_offsets[g+1] belong to one workflow, whose
    makespans count up to limits[g]; answer a holds the tokens
    offsets[a]..offsets[a+1].  mean: "tokens" or "sequences"."""
    c = _Call("sched_group_advantages", makespans, stream)
    t = c.tokens(tokens)
    if mean not in _MEANS:
        _refuse(-3, c.where + ": mean is 'tokens' or 'sequences'")
    n, g = makespans.numel(), limits.numel()
    advantages, weights = c.floats(advantages, t.n), c.floats(weights, t.n)
    ws, at, nbytes = c.workspace(workspace, 4 * n)
    c.done("sched_group_advantages", c.vector(makespans, _INT64, n),
           c.vector(limits, _INT64, g), c.vector(group_offsets, _INT32, g + 1), g,
           c.vector(offsets, _INT32, n + 1), n, ctypes.byref(t), _MEANS[mean],
           advantages.data_ptr(), weights.data_ptr(), at, nbytes)
    return advantages, weights


def sched_policy_loss(logits, tokens, old_logp, ref_logp, advantages, weights,
                      clip_low: float = 0.2, clip_high: float = 0.2, kl_weight: float = 0.0,
                      temperature: float = 1.0, loss_scale: float = 1.0, loss=None, losses=None,
                      logp=None, d_logits=None, stream=None):
    """(loss, losses, logp, d_logits) of the clipped policy loss; ref_logp may
    be None where kl_weight is 0, d_logits the logits themselves."""
    c = _Call("sched_policy_loss", logits, stream)
    m, t, f32 = c.matrix(logits), c.tokens(tokens), _F32
    if d_logits is None:
        d_logits = c.new((m.rows, m.cols), logits.dtype)
    loss, losses, logp = c.floats(loss, 1), c.floats(losses, t.n), c.floats(logp, t.n)
    d = sched_policy_desc(
        m, t, c.vector(old_logp, f32, t.n),
        None if ref_logp is None else c.vector(ref_logp, f32, t.n),
        c.vector(advantages, f32, t.n), c.vector(weights, f32, t.n), clip_low, clip_high,
        kl_weight, temperature, loss_scale, loss.data_ptr(), losses.data_ptr(), logp.data_ptr(),
        c.matrix(d_logits))
    c.done("sched_policy_loss", ctypes.byref(d))
    return loss, losses, logp, d_logits


def sched_preference_loss(logp, ref_logp, tokens, offsets, beta: float = 0.1,
                          smoothing: float = 0.0, loss_scale: float = 1.0, loss=None, margins=None,
                          d_logp=None, stream=None):
    """(loss, margins, d_logp) over pairs: sequence 2p of offsets is the better
    mapping's, 2p + 1 the worse one's."""
    c = _Call("sched_preference_loss", logp, stream)
    t = c.tokens(tokens)
    pairs, odd = divmod(offsets.numel() - 1, 2)
    if odd:
        _refuse(-2, c.where + ": two sequences per pair")
    loss, margins, d_logp = c.floats(loss, 1), c.floats(margins, pairs), c.floats(d_logp, t.n)
    c.done("sched_preference_loss", c.vector(logp, _F32, t.n), c.vector(ref_logp, _F32, t.n),
           ctypes.byref(t), c.vector(offsets, _INT32), pairs, beta, smoothing, loss_scale,
           loss.data_ptr(), margins.data_ptr(), d_logp.data_ptr())
    return loss, margins, d_logp


def _heads(c: _Call, t, dtype, heads: int, dim: int) -> Tuple:
    if c.other or t.get_device() != c.index:
        c.use(t)
    if t.dtype is not dtype:
        _refuse(-3, c.where + ": tensors of one type")
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        _refuse(-2, f"{c.where}: rows x {heads} heads x {dim}")
    a, b, e = t.stride()
    if e != 1 and dim > 1:
        _refuse(-3, c.where + ": the elements of a head are next to each other")
    return t.data_ptr(), a, b


def _attention_values(c, q, k, v, out, lse, q_offsets, k_offsets, k_lengths, causal, scale):
    if q.dim() != 3 or k.dim() != 3 or k.shape[0] != v.shape[0]:
        _refuse(-2, c.where + ": q, k and v are rows x heads x dim")
    rows, heads, dim = q.shape
    k_rows, kv_heads, _ = k.shape
    dtype, n = q.dtype, q_offsets.numel() - 1
    values = (
        *_heads(c, q, dtype, heads, dim), *_heads(c, k, dtype, kv_heads, dim),
        *_heads(c, v, dtype, kv_heads, dim), *_heads(c, out, dtype, heads, dim),
        c.vector(lse, _F32, heads * rows), _types.get(dtype, -1), dim, heads, kv_heads, rows, k_rows,
        c.vector(q_offsets, _INT32), c.vector(k_offsets, _INT32, n + 1),
        0 if k_lengths is None else c.vector(k_lengths, _INT32, n), n, int(causal),
        1.0 / math.sqrt(max(dim, 1)) if scale is None else scale)
    if out.shape[0] != rows:
        _refuse(-2, c.where + ": out has a row per query")
    return values


def sched_attention(q, k, v, q_offsets, k_offsets, k_lengths=None, causal: bool = True,
                    scale: Optional[float] = None, out=None, lse=None, workspace=None,
                    stream=None) -> Tuple:
    """(out, lse) of packed sequences: q is rows x q_heads x dim, k and v rows x
    kv_heads x dim (slices of one projection, or cache slots with k_lengths);
    lse is q_heads x rows.  scale: 1 / sqrt(dim) unless it is given."""
    c = _Call("sched_attention", q, stream)
    if out is None:
        out = c.like_of(q)
    if lse is None:
        lse = c.new((q.shape[1], q.shape[0]) if q.dim() == 3 else (0,), _F32)
    d = c.packed(_pack_attention, _attention_values(c, q, k, v, out, lse, q_offsets, k_offsets,
                                                    k_lengths, causal, scale))
    need = c.bytes("sched_attention_workspace_bytes", d)
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_attention", d, at, nbytes)
    return out, lse


def sched_attention_grad(q, k, v, out, lse, d_out, q_offsets, k_offsets, k_lengths=None,
                         causal: bool = True, scale: Optional[float] = None, d_q=None, d_k=None,
                         d_v=None, workspace=None, stream=None) -> Tuple:
    """(d_q, d_k, d_v) from sched_attention's arguments and results and d_out."""
    c = _Call("sched_attention_grad", q, stream)
    d = c.packed(_pack_attention, _attention_values(c, q, k, v, out, lse, q_offsets, k_offsets,
                                                    k_lengths, causal, scale))
    grads = []
    for given, like in ((d_q, q), (d_k, k), (d_v, v)):
        t = c.like_of(like) if given is None else given
        if t.shape[0] != like.shape[0]:
            _refuse(-2, c.where + ": a gradient has its tensor's rows")
        grads.append(t)
    if d_out.shape[0] != q.shape[0]:
        _refuse(-2, c.where + ": d_out has a row per query")
    g = [_pack_heads(*_heads(c, t, q.dtype, like.shape[1], q.shape[2]))
         for t, like in zip((d_out, *grads), (q, q, k, v))]
    need = c.bytes("sched_attention_grad_workspace_bytes", d)
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_attention_grad", d, *g, at, nbytes)
    return tuple(grads)


def _shared_desc(c, q, k, v, prefix_k, prefix_v, out, lse, q_offsets, k_offsets, prefix_offsets,
                 group_offsets, k_lengths, prefix_lengths, causal, scale):
    own = _attention_values(c, q, k, v, out, lse, q_offsets, k_offsets, k_lengths, causal, scale)
    if prefix_k.dim() != 3 or prefix_k.shape[0] != prefix_v.shape[0]:
        _refuse(-2, c.where + ": the prefix' keys and values are rows x heads x dim")
    kv, dim, dtype, groups = k.shape[1], k.shape[2], q.dtype, group_offsets.numel() - 1
    return c.packed(_pack_shared, (
        *own, *_heads(c, prefix_k, dtype, kv, dim), *_heads(c, prefix_v, dtype, kv, dim),
        prefix_k.shape[0], c.vector(prefix_offsets, _INT32, groups + 1),
        0 if prefix_lengths is None else c.vector(prefix_lengths, _INT32, groups),
        c.vector(group_offsets, _INT32), groups))


def sched_shared_attention(q, k, v, prefix_k, prefix_v, q_offsets, k_offsets, prefix_offsets,
                           group_offsets, k_lengths=None, prefix_lengths=None, causal: bool = True,
                           scale: Optional[float] = None, out=None, lse=None, workspace=None,
                           stream=None) -> Tuple:
    """(out, lse) as sched_attention, where the sequences group_offsets[g] ..
    group_offsets[g+1] see the prefix rows prefix_offsets[g] ..
    prefix_offsets[g+1] (the first prefix_lengths[g]) before their own keys."""
    c = _Call("sched_shared_attention", q, stream)
    if out is None:
        out = c.like_of(q)
    if lse is None:
        lse = c.new((q.shape[1], q.shape[0]) if q.dim() == 3 else (0,), _F32)
    d = _shared_desc(c, q, k, v, prefix_k, prefix_v, out, lse, q_offsets, k_offsets, prefix_offsets,
                     group_offsets, k_lengths, prefix_lengths, causal, scale)
    need = c.bytes("sched_shared_attention_workspace_bytes", d)
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_shared_attention", d, at, nbytes)
    return out, lse


def sched_shared_attention_grad(q, k, v, prefix_k, prefix_v, out, lse, d_out, q_offsets, k_offsets,
                                prefix_offsets, group_offsets, k_lengths=None, prefix_lengths=None,
                                causal: bool = True, scale: Optional[float] = None, d_q=None,
                                d_k=None, d_v=None, d_prefix_k=None, d_prefix_v=None,
                                workspace=None, stream=None) -> Tuple:
    """(d_q, d_k, d_v, d_prefix_k, d_prefix_v) from sched_shared_attention's
    arguments and results and d_out."""
    c = _Call("sched_shared_attention_grad", q, stream)
    d = _shared_desc(c, q, k, v, prefix_k, prefix_v, out, lse, q_offsets, k_offsets, prefix_offsets,
                     group_offsets, k_lengths, prefix_lengths, causal, scale)
    likes = (q, k, v, prefix_k, prefix_v)
    grads = []
    for given, like in zip((d_q, d_k, d_v, d_prefix_k, d_prefix_v), likes):
        t = c.like_of(like) if given is None else given
        if t.shape[0] != like.shape[0]:
            _refuse(-2, c.where + ": a gradient has its tensor's rows")
        grads.append(t)
    if d_out.shape[0] != q.shape[0]:
        _refuse(-2, c.where + ": d_out has a row per query")
    values = []
    for t, like in zip((d_out, *grads), (q, *likes)):
        values += _heads(c, t, q.dtype, like.shape[1], q.shape[2])
    need = c.bytes("sched_shared_attention_grad_workspace_bytes", d)
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_shared_attention_grad", d, _pack_grads(*values), at, nbytes)
    return tuple(grads)


def _rotate_desc(c, q, k, positions, frequencies, q_weight, k_weight, places, out_rows, norm, eps,
                 interleaved, outs=None):
    """outs: (v or None, q_out, k_out, v_out or None) of the forward pass."""
    if q.dim() != 3 or k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        _refuse(-2, c.where + ": q and k are rows x heads x dim")
    rows, heads, dim = q.shape
    kv, dtype = k.shape[1], q.dtype
    turned = 2 * frequencies.numel() if frequencies is not None else 0
    to = _NOWHERE
    if places is not None:
        to = c.token_values(places)
        if rows == 0:  # an empty tensor has no address
            to = (256, *to[1:])
    else:
        out_rows = rows
    v = q_out = k_out = v_out = _NO_HEADS
    if outs is not None:
        if outs[1].shape[0] != rows or outs[2].shape[0] != out_rows:
            _refuse(-2, c.where + ": outputs have a row per input row")
        q_out, k_out = _heads(c, outs[1], dtype, heads, dim), _heads(c, outs[2], dtype, kv, dim)
        if outs[0] is not None:
            if outs[0].shape[0] != rows or outs[3].shape[0] != out_rows:
                _refuse(-2, c.where + ": v has k's rows")
            v, v_out = _heads(c, outs[0], dtype, kv, dim), _heads(c, outs[3], dtype, kv, dim)
    return c.packed(_pack_rotate, (
        *_heads(c, q, dtype, heads, dim), *_heads(c, k, dtype, kv, dim), *v, *q_out, *k_out, *v_out,
        _types.get(dtype, -1), dim, heads, kv, rows, out_rows, *c.token_values(positions), *to,
        0 if q_weight is None else c.vector(q_weight, _F32, dim),
        0 if k_weight is None else c.vector(k_weight, _F32, dim),
        c.vector(frequencies, _F32) if turned else 0, turned, int(interleaved), int(norm), eps))


def sched_norm_rotate(q, k, positions, frequencies, q_weight=None, k_weight=None, v=None,
                      places=None, norm: bool = True, eps: float = 1e-6, interleaved: bool = False,
                      q_out=None, k_out=None, v_out=None, stream=None) -> Tuple:
    """(q_out, k_out), and v_out where v is given: heads normed, weighted and
    turned by their rows' positions (int32 or int64) times `frequencies`
    (float32, one per pair; None: not turned).  With `places` row i of k and v
    goes to that row of k_out and v_out (caches, which are given)."""
    c = _Call("sched_norm_rotate", q, stream)
    if places is not None and (k_out is None or (v is not None and v_out is None)):
        _refuse(-1, c.where + ": places are rows of a given k_out and v_out")
    if q_out is None:
        q_out = c.like_of(q)
    if k_out is None:
        k_out = c.like_of(k)
    if v is not None and v_out is None:
        v_out = c.like_of(v)
    d = _rotate_desc(c, q, k, positions, frequencies, q_weight, k_weight, places, k_out.shape[0], norm,
                     eps, interleaved, (v, q_out, k_out, v_out))
    c.done("sched_norm_rotate", d)
    return (q_out, k_out) if v is None else (q_out, k_out, v_out)


def sched_norm_rotate_grad(q, k, d_q_out, d_k_out, positions, frequencies, q_weight=None,
                           k_weight=None, places=None, norm: bool = True, eps: float = 1e-6,
                           interleaved: bool = False, d_q=None, d_k=None, d_q_weight=None,
                           d_k_weight=None, workspace=None, stream=None) -> Tuple:
    """(d_q, d_k, d_q_weight, d_k_weight) from sched_norm_rotate's inputs and
    the gradients of its results; of a weight that is not given None."""
    c = _Call("sched_norm_rotate_grad", q, stream)
    d = _rotate_desc(c, q, k, positions, frequencies, q_weight, k_weight, places, d_k_out.shape[0],
                     norm, eps, interleaved)
    rows, heads, dim = q.shape
    if d_q is None:
        d_q = c.like_of(q)
    if d_k is None:
        d_k = c.like_of(k)
    if d_q_weight is None and q_weight is not None:
        d_q_weight = c.new((dim,), _F32)
    if d_k_weight is None and k_weight is not None:
        d_k_weight = c.new((dim,), _F32)
    if d_q_out.shape[0] != rows or d_q.shape[0] != rows or d_k.shape[0] != rows or (
            places is None and d_k_out.shape[0] != rows):
        _refuse(-2, c.where + ": a gradient has its tensor's rows")
    h = [_pack_heads(*_heads(c, t, q.dtype, n, dim))
         for t, n in ((d_q_out, heads), (d_k_out, k.shape[1]), (d_q, heads), (d_k, k.shape[1]))]
    w = [None if t is None else c.vector(t, _F32, dim) for t in (d_q_weight, d_k_weight)]
    need = c.bytes("sched_norm_rotate_grad_workspace_bytes", d)
    ws, at, nbytes = c.workspace(workspace, need if any(w) else 0)
    c.done("sched_norm_rotate_grad", d, *h, *w, at, nbytes)
    return d_q, d_k, d_q_weight, d_k_weight


def sched_beam_select(logits, scores, beams: int, width: Optional[int] = None, last=None,
                      end_token: int = -1, temperature: float = 1.0, stay: bool = False,
                      new_scores=None, parents=None, tokens=None, workspace=None,
                      stream=None) -> Tuple:
    """(new_scores, parents, tokens) of the `width` (default: beams) best
    continuations of each group of `beams` rows: float32, int32 row of the
    parent, and int64 (or as `tokens` is).  `last` has the beams' last tokens; a
    beam that ends in end_token is finished.  stay: a beam's best continuation
    keeps its slot; otherwise results are ordered by score."""
    c = _Call("sched_beam_select", logits, stream)
    m = c.matrix_values(logits)
    rows, width = m[2], beams if width is None else width
    if not (1 <= beams <= 128 and 1 <= width <= 128) or rows % beams:
        _refuse(-2, c.where + ": a row per beam, 1 to 128 beams and results")
    groups = rows // beams
    n = groups * width
    if new_scores is None:
        new_scores = c.new((n,), _F32)
    if parents is None:
        parents = c.new((n,), _INT32)
    if tokens is None:
        tokens = c.new((n,), _INT64)
    at, bits, count = c.token_values(tokens)
    if count != n:
        _refuse(-2, f"{c.where}: {n} tokens, not {count}")
    d = c.packed(_pack_beam, (
        *m, c.vector(scores, _F32, rows),
        *(_NOWHERE if last is None else c.token_values(last)), end_token, groups, beams, width,
        int(stay), temperature, c.vector(new_scores, _F32, n), c.vector(parents, _INT32, n), at, bits))
    need = c.bytes("sched_beam_workspace_bytes", d)
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_beam_select", d, at, nbytes)
    return new_scores, parents, tokens


def sched_beam_reorder(states, parents, beams: int, lengths=None, stream=None):
    """Slot s of states (outer x slots x rows x ..., a row's elements next to
    each other) gets the first lengths[p] rows (None: all) of slot p =
    parents[s] of its group of `beams`, in place; returns states."""
    c = _Call("sched_beam_reorder", states, stream)
    c.use(states)
    if states.dim() < 3 or not 1 <= beams <= 128:
        _refuse(-2, c.where + ": states are outer x slots x rows x ..., 1 to 128 beams")
    size, row, shape, steps = states.element_size(), 1, states.shape, states.stride()
    for i in range(len(shape) - 1, 2, -1):
        if shape[i] != 1 and steps[i] != row:
            _refuse(-3, c.where + ": the elements of a row are next to each other")
        row *= shape[i]
    slots = shape[1]
    d = c.packed(_pack_states, (states.data_ptr(), shape[0], slots, shape[2], row * size, steps[0] * size,
                                steps[1] * size, steps[2] * size))
    c.done("sched_beam_reorder", d, c.vector(parents, _INT32, slots),
           None if lengths is None else c.vector(lengths, _INT32, slots), beams)
    return states
