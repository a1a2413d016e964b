"""The C ABI of include/sched_policy.h on the host: exported symbols, and what
is refused before any device work."""
import ctypes
import math
import os
import re

import pytest

import paper_2607_22242_amd as S
from paper_2607_22242_amd import binding as B
from paper_2607_22242_amd import policy as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sched_policy.h")
NULL, SIZE, VALUE, WORKSPACE = -1, -2, -3, -8
FAKE = 1 << 20  # never dereferenced: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    L = B.lib()
    for name, args in P._ARGS.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = ctypes.c_int, args
    return L


def test_library_exports_every_declared_function(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sched_[a-z_]+)\s*\(", text)))
    assert names == sorted(P.POLICY_EXPORTED) == sorted(P._ARGS)
    for name in names:
        assert hasattr(lib, name), name
    assert not set(names) & set(B.EXPORTED)


def matrix(rows=4, cols=10, dtype=0, data=FAKE, stride=None):
    return P.sched_matrix(data, dtype, rows, cols, cols if stride is None else stride)


def tokens(n=4, bits=64, data=FAKE):
    return P.sched_tokens(data, bits, n)


R = ctypes.byref


def test_embed(lib):
    def rc(table=None, tok=None, out=None, scale=1.0):
        return lib.sched_embed(R(table or matrix(7)), R(tok or tokens()), scale, R(out or matrix()), 0)
    assert lib.sched_embed(None, R(tokens()), 1.0, R(matrix()), 0) == NULL
    assert rc(table=matrix(7, data=0)) == NULL
    assert rc(table=matrix(-1)) == SIZE
    assert rc(table=matrix(7, 11)) == SIZE
    assert rc(table=matrix(7, dtype=3)) == VALUE
    assert rc(table=matrix(7, dtype=1)) == VALUE            # another type than out's
    assert rc(table=matrix(7, data=FAKE + 2)) == VALUE      # a float at 2 bytes
    assert rc(tok=tokens(3)) == SIZE
    assert rc(tok=tokens(bits=16)) == VALUE
    assert rc(tok=tokens(data=FAKE + 4)) == VALUE
    assert rc(tok=tokens(data=0)) == NULL
    assert rc(out=matrix(stride=9)) == VALUE                # rows that overlap
    assert rc(scale=math.inf) == VALUE
    # nothing to do is no error, and starts nothing
    assert lib.sched_embed(R(matrix(7)), R(tokens(0, data=0)), 1.0, R(matrix(0, data=0)), 0) == 0


def test_embed_grad(lib):
    need = ctypes.c_size_t()
    assert lib.sched_embed_grad_workspace_bytes(4, 10, None) == NULL
    assert lib.sched_embed_grad_workspace_bytes(-1, 10, R(need)) == SIZE
    assert lib.sched_embed_grad_workspace_bytes(4, 1 << 25, R(need)) == SIZE
    assert lib.sched_embed_grad_workspace_bytes(4, 10, R(need)) == 0 and need.value >= 32

    def rc(rows=None, out=None, add=0, ws=FAKE, size=need.value):
        return lib.sched_embed_grad(R(rows or matrix()), R(tokens()), 1.0, add, R(out or matrix(7)), ws,
                                    size, 0)
    assert rc(rows=matrix(3)) == SIZE
    assert rc(out=matrix(7, 9)) == SIZE
    assert rc(out=matrix(7, dtype=2)) == VALUE
    assert rc(add=2) == VALUE
    assert rc(ws=0) == WORKSPACE
    assert rc(ws=FAKE + 128) == WORKSPACE
    assert rc(size=need.value - 1) == WORKSPACE


def test_logprobs(lib):
    def rc(x=None, t=None, temperature=1.0, logp=FAKE):
        return lib.sched_token_logprobs(R(x or matrix()), R(t or tokens()), temperature, logp, 0)
    assert rc(logp=0) == NULL
    assert rc(x=matrix(3)) == SIZE
    assert rc(x=matrix(4, 0)) == SIZE
    assert rc(x=matrix(4, 1 << 32)) == SIZE
    for bad in (0.0, -1.0, math.nan, math.inf, 1e-45):
        assert rc(temperature=bad) == VALUE
    x, t = matrix(), tokens()
    g = lambda d: lib.sched_token_logprobs_grad(R(x), R(t), 1.0, FAKE, FAKE, R(d), 0)  # noqa: E731
    assert g(matrix(3)) == SIZE
    assert g(matrix(dtype=1)) == VALUE
    assert g(matrix(stride=11)) == VALUE                    # in place, with other rows
    assert lib.sched_token_logprobs_grad(R(x), R(t), 1.0, 0, FAKE, R(matrix()), 0) == NULL


def test_losses(lib):
    def policy(**kw):
        a = dict(logits=matrix(), tokens=tokens(), old_logp=FAKE, ref_logp=FAKE, advantages=FAKE,
                 weights=FAKE, clip_low=0.2, clip_high=0.2, kl_weight=0.1, temperature=1.0,
                 loss_scale=1.0, loss=FAKE, losses=FAKE, logp=FAKE, d_logits=matrix(data=FAKE * 2))
        a.update(kw)
        return lib.sched_policy_loss(R(P.sched_policy_desc(*a.values())), 0)
    assert lib.sched_policy_loss(None, 0) == NULL
    for name in ("old_logp", "ref_logp", "advantages", "weights", "loss", "losses", "logp"):
        assert policy(**{name: 0}) == NULL, name
    for name in ("clip_low", "clip_high"):
        for bad in (-0.1, math.nan, math.inf):
            assert policy(**{name: bad}) == VALUE
    for name in ("kl_weight", "loss_scale"):
        assert policy(**{name: math.nan}) == VALUE
    assert policy(temperature=0.0) == VALUE
    assert policy(d_logits=matrix(5)) == SIZE

    def pairs(n=1, beta=0.1, eps=0.0, offsets=FAKE, loss=FAKE, logp=FAKE):
        return lib.sched_preference_loss(logp, FAKE, R(tokens()), offsets, n, beta, eps, 1.0, loss, FAKE,
                                         FAKE, 0)
    assert pairs(0) == SIZE and pairs(1 << 23) == SIZE
    assert pairs(beta=math.inf) == VALUE
    assert pairs(eps=-0.1) == pairs(eps=1.1) == pairs(eps=math.nan) == VALUE
    assert pairs(offsets=0) == pairs(loss=0) == pairs(logp=0) == NULL

    def advantages(n=3, g=1, mean=0, ws=FAKE, size=12, limit=FAKE, out=FAKE):
        return lib.sched_group_advantages(FAKE, limit, FAKE, g, FAKE, n, R(tokens()), mean, out, FAKE,
                                          ws, size, 0)
    assert advantages(n=-1) == advantages(n=1 << 24) == advantages(g=0) == SIZE
    assert advantages(mean=2) == VALUE
    assert advantages(limit=0) == advantages(out=0) == NULL
    assert advantages(size=11) == advantages(ws=0) == WORKSPACE


def test_most_answers_and_rows(lib):
    def advantages(n, ws):
        return lib.sched_group_advantages(FAKE, FAKE, FAKE, 1, FAKE, n, R(tokens()), 0, FAKE, FAKE,
                                          ws, 0, 0)
    assert advantages((1 << 16) + 1, FAKE) == SIZE and advantages(1 << 16, FAKE) == WORKSPACE
    rows = (1 << 31) - 1023
    assert lib.sched_embed_grad_workspace_bytes(rows, 8, R(ctypes.c_size_t())) == SIZE
    assert lib.sched_embed_grad_workspace_bytes(rows - 1, 8, R(ctypes.c_size_t())) == 0


def test_attention(lib):
    def desc(**kw):
        h = P.sched_heads(FAKE, 256, 64)
        a = dict(q=h, k=P.sched_heads(FAKE, 128, 64), v=P.sched_heads(FAKE, 128, 64), out=h, lse=FAKE,
                 dtype=2, head_dim=64, q_heads=4, kv_heads=2, q_rows=6, k_rows=6, q_offsets=FAKE,
                 k_offsets=FAKE, k_lengths=0, n_seqs=1, causal=1, scale=0.1)
        a.update(kw)
        return P.sched_attention_desc(*a.values())
    rc = lambda **kw: lib.sched_attention(R(desc(**kw)), FAKE, 1 << 30, 0)  # noqa: E731
    assert lib.sched_attention(None, FAKE, 0, 0) == NULL
    for bad in (dict(head_dim=0), dict(head_dim=136), dict(head_dim=20), dict(q_heads=3),
                dict(kv_heads=0), dict(q_rows=-1), dict(k_rows=1 << 31), dict(n_seqs=-1),
                dict(q_rows=1 << 31), dict(q_heads=8194, kv_heads=2), dict(n_seqs=1 << 24)):
        assert rc(**bad) == SIZE, bad
    for bad in (dict(dtype=0), dict(dtype=7), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                dict(causal=2), dict(q=P.sched_heads(FAKE + 8, 256, 64)),
                dict(k=P.sched_heads(FAKE, 132, 64)), dict(v=P.sched_heads(FAKE, 128, 68)),
                dict(q=P.sched_heads(FAKE, -256, 64)),
                dict(out=P.sched_heads(FAKE, 128, 64)),     # heads of rows that overlap
                dict(out=P.sched_heads(FAKE, 256, 32))):
        assert rc(**bad) == VALUE, bad
    for bad in (dict(q=P.sched_heads(0, 256, 64)), dict(lse=0), dict(q_offsets=0), dict(k_offsets=0)):
        assert rc(**bad) == NULL, bad
    need = ctypes.c_size_t()
    long = dict(k_rows=1 << 20, k=P.sched_heads(FAKE, 128, 64))
    assert lib.sched_attention_workspace_bytes(R(desc(**long)), R(need)) == 0 and need.value > 0
    assert lib.sched_attention(R(desc(**long)), FAKE, need.value - 1, 0) == WORKSPACE
    assert lib.sched_attention_workspace_bytes(R(desc(head_dim=7)), R(need)) == SIZE
    q, k = P.sched_heads(FAKE, 256, 64), P.sched_heads(FAKE, 128, 64)
    grad = lambda *h, ws=FAKE, size=1 << 20: lib.sched_attention_grad(  # noqa: E731
        R(desc()), *[None if x is None else R(x) for x in h], ws, size, 0)
    assert lib.sched_attention_grad_workspace_bytes(R(desc()), R(need)) == 0
    assert grad(None, q, k, k) == NULL
    assert grad(q, q, P.sched_heads(0, 128, 64), k) == NULL
    assert grad(q, k, k, k) == VALUE                        # d_q's heads overlap
    assert grad(q, q, k, k, size=need.value - 1) == WORKSPACE
    assert grad(q, q, k, k, ws=FAKE + 8) == WORKSPACE


def test_binding_refuses_tensors_of_the_host():
    torch = pytest.importorskip("torch")
    x, t = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: S.sched_embed(x, t), lambda: S.sched_token_logprobs(x, t),
                 lambda: S.sched_attention(x, x, x, t, t), lambda: S.sched_embed_grad(x, t, 9)):
        with pytest.raises(S.SchedError) as e:
            call()
        assert e.value.name == "SCHED_E_VALUE"


def test_temperatures_whose_factors_leave_32_bits(lib):
    """log2(e) / temperature is what the rows are multiplied with: refused where
    it is infinite, though 1 / temperature is not."""
    for t in (3.5e-39, 4.0e-39, 2.94e-39):
        assert 1.0 / t < 3.4028e38 < math.log2(math.e) / t
        assert lib.sched_token_logprobs(R(matrix()), R(tokens()), t, FAKE, 0) == VALUE
        desc = P.sched_policy_desc(matrix(), tokens(), FAKE, FAKE, FAKE, FAKE, 0.2, 0.2, 0.0, t, 1.0, FAKE,
                                   FAKE, FAKE, matrix(data=FAKE * 2))
        assert lib.sched_policy_loss(R(desc), 0) == VALUE
