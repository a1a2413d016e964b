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
from typing import Optional, Tuple

from . import binding as _b
from .binding import SchedError

POLICY_EXPORTED = ["sched_embed", "sched_embed_grad_workspace_bytes", "sched_embed_grad",
                   "sched_token_logprobs", "sched_token_logprobs_grad", "sched_group_advantages",
                   "sched_policy_loss", "sched_preference_loss",
                   "sched_attention_workspace_bytes", "sched_attention",
                   "sched_attention_grad_workspace_bytes", "sched_attention_grad"]

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
}

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

    __slots__ = ("where", "device", "index", "stream", "ptr", "other")

    def __init__(self, where: str, first, stream):
        if _torch is None:
            _load()
        self.where = where
        index = first.get_device() if isinstance(first, _torch.Tensor) else -1
        if index < 0 or not first.is_cuda:
            _refuse(-3, where + ": tensors are on a GPU")
        self.index, self.device, self.stream = index, first.device, stream
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
            return _torch.empty(shape, dtype=dtype, device=self.device)
        with _torch.cuda.stream(self.stream):
            return _torch.empty(shape, dtype=dtype, device=self.device)

    def matrix(self, t) -> sched_matrix:
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
        return sched_matrix(t.data_ptr(), kind, rows, cols, stride)

    def tokens(self, t) -> sched_tokens:
        self.use(t)
        bits = 64 if t.dtype == _INT64 else 32 if t.dtype == _INT32 else 0
        if not bits or not t.is_contiguous():
            _refuse(-3, self.where + ": tokens are contiguous int32 or int64")
        return sched_tokens(t.data_ptr(), bits, t.numel())

    def vector(self, t, dtype, n: Optional[int] = None) -> int:
        self.use(t)
        if t.dtype != dtype or not t.is_contiguous():
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


def _heads(c: _Call, t, dtype, heads: int, dim: int) -> sched_heads:
    c.use(t)
    if t.dtype != dtype:
        _refuse(-3, c.where + ": tensors of one type")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != dim:
        _refuse(-2, f"{c.where}: rows x {heads} heads x {dim}")
    a, b, e = t.stride()
    if e != 1 and dim > 1:
        _refuse(-3, c.where + ": the elements of a head are next to each other")
    return sched_heads(t.data_ptr(), a, b)


def _attention_desc(c, q, k, v, out, lse, q_offsets, k_offsets, k_lengths, causal, scale):
    if q.dim() != 3 or k.dim() != 3 or k.shape[0] != v.shape[0]:
        _refuse(-2, c.where + ": q, k and v are rows x heads x dim")
    rows, heads, dim = q.shape
    n = q_offsets.numel() - 1
    d = sched_attention_desc(
        _heads(c, q, q.dtype, heads, dim), _heads(c, k, q.dtype, k.shape[1], dim),
        _heads(c, v, q.dtype, k.shape[1], dim), _heads(c, out, q.dtype, heads, dim),
        c.vector(lse, _F32, heads * rows), _types.get(q.dtype, -1), dim, heads,
        k.shape[1], rows, k.shape[0], c.vector(q_offsets, _INT32),
        c.vector(k_offsets, _INT32, n + 1),
        None if k_lengths is None else c.vector(k_lengths, _INT32, n), n, int(causal),
        1.0 / math.sqrt(max(dim, 1)) if scale is None else scale)
    if out.shape[0] != rows:
        _refuse(-2, c.where + ": out has a row per query")
    return d


def sched_attention(q, k, v, q_offsets, k_offsets, k_lengths=None, causal: bool = True,
                    scale: Optional[float] = None, out=None, lse=None, workspace=None,
                    stream=None) -> Tuple:
    """(out, lse) of packed sequences: q is rows x q_heads x dim, k and v rows x
    kv_heads x dim (slices of one projection, or cache slots with k_lengths);
    lse is q_heads x rows.  scale: 1 / sqrt(dim) unless it is given."""
    c = _Call("sched_attention", q, stream)
    if out is None:
        out = c.new(tuple(q.shape), q.dtype)
    if lse is None:
        lse = c.new((q.shape[1], q.shape[0]) if q.dim() == 3 else (0,), _F32)
    d = _attention_desc(c, q, k, v, out, lse, q_offsets, k_offsets, k_lengths, causal, scale)
    need = c.bytes("sched_attention_workspace_bytes", ctypes.byref(d))
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_attention", ctypes.byref(d), at, nbytes)
    return out, lse


def sched_attention_grad(q, k, v, out, lse, d_out, q_offsets, k_offsets, k_lengths=None,
                         causal: bool = True, scale: Optional[float] = None, d_q=None, d_k=None,
                         d_v=None, workspace=None, stream=None) -> Tuple:
    """(d_q, d_k, d_v) from sched_attention's arguments and results and d_out."""
    c = _Call("sched_attention_grad", q, stream)
    d = _attention_desc(c, q, k, v, out, lse, q_offsets, k_offsets, k_lengths, causal, scale)
    grads = []
    for given, like in ((d_q, q), (d_k, k), (d_v, v)):
        t = c.new(tuple(like.shape), q.dtype) if given is None else given
        if t.shape[0] != like.shape[0]:
            _refuse(-2, c.where + ": a gradient has its tensor's rows")
        grads.append(t)
    if d_out.shape[0] != q.shape[0]:
        _refuse(-2, c.where + ": d_out has a row per query")
    do = _heads(c, d_out, q.dtype, q.shape[1], q.shape[2])
    g = [_heads(c, t, q.dtype, like.shape[1], q.shape[2]) for t, like in zip(grads, (q, k, v))]
    need = c.bytes("sched_attention_grad_workspace_bytes", ctypes.byref(d))
    ws, at, nbytes = c.workspace(workspace, need)
    c.done("sched_attention_grad", ctypes.byref(d), ctypes.byref(do), ctypes.byref(g[0]),
           ctypes.byref(g[1]), ctypes.byref(g[2]), at, nbytes)
    return tuple(grads)
