"""The operators of include/sched_policy.h that serve many answers to one
prompt, against plain 64-bit forms (answers64), element by element within the
bounds that their roundings give."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import answers64 as R  # noqa: E402
from policy64 import close  # noqa: E402

import paper_2607_22242_amd as S  # noqa: E402

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# --- norms and rotation --------------------------------------------------------


def check_rotate(g, rows, hq, hk, dim, turned, dtype, interleaved=False, norm=True, weights=True,
                 far=4096, eps=1e-6, bits=torch.int64):
    x = randn(g, rows, hq + 2 * hk, dim, dtype=dtype)
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    w = [1 + 0.2 * randn(g, dim) if weights and norm else None for _ in range(2)]
    freq = 10000.0 ** (-torch.arange(turned // 2) / max(1, turned // 2))
    pos = torch.randint(-far, far + 1, (rows,), generator=g)
    do = [randn(g, rows, h, dim, dtype=dtype) for h in (hq, hk)]
    how = dict(norm=norm, eps=eps, interleaved=interleaved)
    want = [R.Rotate(t, pos, freq, wt, norm, eps, interleaved, d) for t, wt, d in zip((q, k), w, do)]
    d = x.cuda()
    dq, dk, dv = d[:, :hq], d[:, hq:hq + hk], d[:, hq + hk:]
    weight = dict(zip(("q_weight", "k_weight"), [None if t is None else t.cuda() for t in w]))
    at, f = pos.to(bits).cuda(), freq.cuda() if turned else None
    q_out, k_out, v_out = S.sched_norm_rotate(dq, dk, at, f, v=dv, **weight, **how)
    close(q_out, want[0].out, want[0].out_b, "q")
    close(k_out, want[1].out, want[1].out_b, "k")
    assert torch.equal(v_out.cpu(), v)
    grads = S.sched_norm_rotate_grad(dq, dk, do[0].cuda(), do[1].cuda(), at, f, **weight, **how)
    close(grads[0], want[0].dx, want[0].dx_b, "d_q")
    close(grads[1], want[1].dx, want[1].dx_b, "d_k")
    for got, x64 in zip(grads[2:], want):
        if weights and norm:
            close(got, x64.dw, x64.dw_b, "d_weight")
        else:
            assert got is None
    # In place, and the gradient in place of its inputs: the same bits.
    a, b = dq.clone(), dk.clone()
    S.sched_norm_rotate(a, b, at, f, **weight, **how, q_out=a, k_out=b)
    assert torch.equal(a, q_out) and torch.equal(b, k_out)
    a, b = do[0].cuda(), do[1].cuda()
    again = S.sched_norm_rotate_grad(dq, dk, a, b, at, f, **weight, **how, d_q=a, d_k=b)
    for x0, x1 in zip(grads, again):
        assert x0 is None or torch.equal(x0, x1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,hq,hk,dim,turned", [
    (1, 1, 1, 8, 8), (1, 4, 2, 32, 32), (3, 3, 1, 16, 6), (5, 8, 2, 40, 40), (7, 4, 4, 40, 20),
    (33, 2, 1, 64, 64), (9, 5, 5, 80, 16), (65, 16, 4, 96, 96), (17, 1, 1, 120, 120), (40, 32, 8, 128, 128),
    (130, 3, 3, 128, 64), (6, 2, 2, 136, 136), (11, 4, 1, 256, 256), (4, 7, 7, 256, 30), (8, 2, 1, 64, 0)])
def test_norm_rotate(dtype, rows, hq, hk, dim, turned):
    g = gen(rows + dim * 3 + turned)
    check_rotate(g, rows, hq, hk, dim, turned, dtype)
    check_rotate(g, rows, hq, hk, dim, turned, dtype, interleaved=True, bits=torch.int32)


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_rotate_without_norms_or_weights(dtype):
    g = gen(3)
    check_rotate(g, 21, 4, 2, 64, 64, dtype, norm=False)
    check_rotate(g, 21, 4, 2, 24, 10, dtype, norm=False, interleaved=True)
    check_rotate(g, 21, 4, 2, 48, 40, dtype, weights=False, eps=0.5)


def test_norm_rotate_of_many_rows():
    """Blocks of one, some and eight rows, whose last ones are not full."""
    for rows in (1023, 2049, 8195, 12001):
        check_rotate(gen(rows), rows, 2, 1, 32, 32, torch.bfloat16)


def test_far_positions_turn_as_well_as_near_ones():
    check_rotate(gen(4), 64, 2, 1, 64, 64, torch.float32, far=(1 << 31) - 1)
    check_rotate(gen(5), 64, 2, 1, 40, 40, torch.float32, far=(1 << 20), interleaved=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_a_cache(dtype):
    """Places in any order, some of them none; what is not written stays; the
    gradient reads the same places."""
    g = gen(8)
    rows, slots = 37, 90
    x, freq = randn(g, rows, 7, 40, dtype=dtype).cuda(), torch.rand(14, generator=g).cuda()
    q, k, v = x[:, :3], x[:, 3:5], x[:, 5:]
    pos = torch.randint(0, 999, (rows,), generator=g).cuda()
    places = torch.randperm(slots, generator=g)[:rows]
    places[5], places[11], places[30] = -1, slots, -7
    q0, k0, v0 = S.sched_norm_rotate(q, k, pos, freq, v=v)
    cache = randn(g, 2, slots, 2, 40, dtype=dtype).cuda()
    kc, vc = cache[0].clone(), cache[1].clone()
    for at in (places.cuda(), places.int().cuda()):
        S.sched_norm_rotate(q, k, pos, freq, v=v, places=at, k_out=kc, v_out=vc)
    want = [cache[0].clone(), cache[1].clone()]
    on = (places >= 0) & (places < slots)
    want[0][places[on].cuda()], want[1][places[on].cuda()] = k0[on.cuda()], v0[on.cuda()]
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])
    d_q, d_cache = randn(g, rows, 3, 40, dtype=dtype).cuda(), randn(g, slots, 2, 40, dtype=dtype).cuda()
    w = torch.ones(40, device="cuda")
    d_k = torch.zeros((rows, 2, 40), dtype=dtype, device="cuda")
    d_k[on.cuda()] = d_cache[places[on].cuda()]
    x[11, 3:5] = float("nan")  # a row without a place, whatever it holds
    a = S.sched_norm_rotate_grad(q, k, d_q, d_cache, pos, freq, w, w, places=places.cuda())
    k = k.clone()
    k[11] = 1
    b = S.sched_norm_rotate_grad(q, k, d_q, d_k, pos, freq, w, w)
    for x0, x1 in zip(a, b):
        assert torch.equal(x0, x1)
    assert not bool(a[1][~on.cuda()].any())


def test_rotation_keeps_products_of_equal_distances():
    """What it is for: a product of a query and a key depends on how far apart
    they are.  Unit heads, 64 pairs: 2^-24 (3.2 + 8 + 4) each, twice."""
    g = gen(12)
    q, k = randn(g, 1, 1, 128), randn(g, 1, 1, 128)
    q, k = q / q.norm(), k / k.norm()
    freq = 500000.0 ** (-torch.arange(64) / 64)
    got = []
    for p in (0, 17, 1 << 20, (1 << 31) - 100):
        a, _ = S.sched_norm_rotate(q.cuda(), k.cuda(), torch.tensor([p + 90], device="cuda"), freq.cuda(), norm=False)
        _, b = S.sched_norm_rotate(q.cuda(), k.cuda(), torch.tensor([p], device="cuda"), freq.cuda(), norm=False)
        got.append(float((a.double() * b.double()).sum()))
    for x in got[1:]:
        assert abs(x - got[0]) < 4 * 16 * 2.0 ** -24


def test_norm_rotate_grad_against_differences():
    g = gen(6)
    q, k, freq = randn(g, 9, 3, 24), randn(g, 9, 2, 24), torch.rand(9, generator=g)
    w, pos = 1 + 0.3 * randn(g, 24), torch.arange(9)
    d_q, d_k = randn(g, 9, 3, 24), randn(g, 9, 2, 24)
    s_q, s_k, s_w = randn(g, 9, 3, 24), randn(g, 9, 2, 24), randn(g, 24)
    got = S.sched_norm_rotate_grad(q.cuda(), k.cuda(), d_q.cuda(), d_k.cuda(), pos.cuda(), freq.cuda(),
                                   w.cuda(), w.cuda(), eps=0.1)

    def loss(h):
        out = 0.0
        for x, sx, d in ((q, s_q, d_q), (k, s_k, d_k)):
            x64, w64 = x.double() + h * sx, w.double() + h * s_w
            n = x64 * (x64.square().mean(-1, keepdim=True) + R.f32(0.1)).rsqrt() * w64
            y, _ = R.rotated(n, pos, freq, False)
            out += float((y * d).sum())
        return out

    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    along = sum(float((a.cpu().double() * b).sum()) for a, b in zip(got, (s_q, s_k, s_w, s_w)))
    # Gradients of order 1 in 32 bits over 1,100 terms of random sign; differences
    # of second order are 1e-10 of their third derivatives.
    assert abs(slope - along) < 1e-4 * max(1.0, abs(slope))


def test_empty_tensors_of_heads():
    x, p = torch.empty((0, 2, 16), device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    f, w = torch.ones(8, device="cuda"), torch.ones(16, device="cuda")
    q, k = S.sched_norm_rotate(x, x, p, f)
    assert q.shape == k.shape == (0, 2, 16)
    cache = torch.ones((4, 2, 16), device="cuda")
    S.sched_norm_rotate(x, x, p, f, places=p, k_out=cache)
    assert bool((cache == 1).all())
    d = S.sched_norm_rotate_grad(x, x, x, x, p, f, w, w)
    assert not bool(d[2].any()) and not bool(d[3].any())


# --- beams ---------------------------------------------------------------------


def check_beams(g, groups, beams, width, vocab, dtype, stay=False, end=-1, temperature=1.0, allowed=1.0,
                dead=0.0, spoil=None, bits=torch.int64):
    n = groups * beams
    for _ in range(60):
        logits = (randn(g, n, vocab) * 2).to(dtype)
        if allowed < 1:
            logits[torch.rand(logits.shape, generator=g) >= allowed] = -math.inf
        scores = -4 - 3 * torch.rand(n, generator=g)
        scores[torch.rand(n, generator=g) < dead] = -math.inf
        last = torch.randint(0, max(vocab, 2), (n,), generator=g)
        if spoil is not None:
            spoil(logits, scores)
        groups64 = R.beam_candidates(logits, scores, beams, last, end, temperature)
        # Scores in 64 bits from sums in 32: errors of some 2^-20 at most.
        if R.apart(groups64, width, 1e-5):
            break
    else:
        raise AssertionError("no input without near ties")
    want = R.beam_results(groups64, beams, width, stay)
    got = S.sched_beam_select(logits.cuda(), scores.cuda(), beams, width, last=last.to(bits).cuda(),
                              end_token=end, temperature=temperature, stay=stay,
                              tokens=torch.empty(groups * width, dtype=bits, device="cuda"))
    assert torch.equal(got[1].cpu().long(), want[1]), "parents"
    assert torch.equal(got[2].cpu().long(), want[2]), "tokens"
    # Powers to 2^-24 (8 spans of their exponents + 4) each, sums of up to 64
    # terms a lane, and the score's own rounding.
    span = max([0.0, *logits[torch.isfinite(logits)].abs().tolist()]) / temperature
    close(got[0], want[0], 2.0 ** -24 * (16 * span + 128 + want[0].nan_to_num(0, 0, 0).abs()), "scores")
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("groups,beams,width,vocab", [
    (1, 1, 1, 1), (2, 1, 3, 2), (3, 4, 4, 3), (13, 64, 64, 3), (2, 128, 128, 5), (5, 3, 7, 40), (1, 16, 16, 256),
    (2, 1, 128, 257), (3, 5, 5, 700), (1, 2, 2, 2047), (2, 3, 3, 2048), (1, 4, 9, 2049), (2, 8, 8, 5003),
    (1, 1, 100, 20001)])
def test_beam_select(dtype, groups, beams, width, vocab):
    g = gen(groups + 7 * beams + vocab)
    check_beams(g, groups, beams, width, vocab, dtype)
    check_beams(g, groups, beams, width, vocab, dtype, end=vocab // 2, temperature=0.7, allowed=0.7,
                dead=0.3, stay=width == beams, bits=torch.int32)


def test_beam_select_of_long_rows():
    check_beams(gen(1), 1, 3, 3, 131077, torch.bfloat16, stay=True)
    check_beams(gen(2), 1, 2, 128, 70001, torch.float32)


def test_beam_select_joins_a_row_s_lists_first():
    """64 beams of 8 strips of 64: more than a block holds."""
    g = gen(9)
    n, vocab = 128, 30011
    logits = torch.randn((n, vocab), generator=g) * 2
    scores = torch.linspace(-4, -9, n)
    got = S.sched_beam_select(logits.cuda(), scores.cuda(), 128, 128)
    z = torch.log_softmax(logits.double(), 1) + scores.double()[:, None]
    best = z.view(-1).topk(129)
    assert float((best.values[:-1] - best.values[1:]).min()) > 1e-6  # of this input: 2^-24 64 steps
    assert torch.equal(got[1].cpu().long(), best.indices[:-1] // vocab)
    assert torch.equal(got[2].cpu(), best.indices[:-1] % vocab)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab,beams,width", [(3, 4, 12), (700, 2, 100), (2048, 1, 128), (9001, 3, 64)])
def test_equal_scores_go_to_the_first(dtype, vocab, beams, width):
    """Rows of one value, and of few: lower beams, then lower tokens first."""
    for values in (1, 3):
        x = (torch.arange(vocab) * 7919 % values).float().expand(beams, vocab).to(dtype).contiguous()
        scores = torch.full((beams,), -2.0)
        groups = R.beam_candidates(x, scores, beams, None, -1, 1.0)
        want = R.beam_results(groups, beams, width, False)
        got = S.sched_beam_select(x.cuda(), scores.cuda(), beams, width)
        assert torch.equal(got[1].cpu().long(), want[1]) and torch.equal(got[2].cpu(), want[2])


@pytest.mark.parametrize("vocab", [40, 5003])
@pytest.mark.parametrize("stay", [False, True])
def test_beams_in_place(vocab, stay):
    g = gen(vocab)
    logits, scores = randn(g, 24, vocab).cuda(), randn(g, 24).cuda()
    last = torch.randint(0, 5, (24,), generator=g).cuda()
    want = S.sched_beam_select(logits, scores, 6, last=last, end_token=2, stay=stay)
    got = S.sched_beam_select(logits, scores, 6, last=last, end_token=2, stay=stay, new_scores=scores, tokens=last)
    assert got[0] is scores and got[2] is last
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_zeros_of_both_signs_are_equal():
    x = torch.tensor([[-0.0, 0.0, -0.0, -1.0]])
    got = S.sched_beam_select(x.cuda(), torch.zeros(1).cuda(), 1, 4)
    assert got[2].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("vocab", [5, 300, 4099])
def test_rows_without_candidates(vocab):
    """Rows of -inf, with NaN or +inf in them, and beams that are not there."""
    def spoil(logits, scores):
        logits[0] = -math.inf
        logits[1, vocab // 2] = math.nan
        logits[2, vocab - 1] = math.inf
        logits[3] = -math.inf
        logits[3, vocab - 1] = math.nan
        scores[4], scores[5], scores[6] = math.nan, math.inf, -math.inf
        logits[8, :-1] = -math.inf

    for stay in (False, True):
        check_beams(gen(vocab), 1, 9, 9, vocab, torch.float32, stay=stay, spoil=spoil)
    # Nothing at all.
    x = torch.full((6, vocab), -math.inf, device="cuda")
    got = S.sched_beam_select(x, torch.zeros(6, device="cuda"), 3, 3, stay=True)
    assert bool((got[0] == -math.inf).all()) and bool((got[1] == -1).all()) and bool((got[2] == -1).all())


def test_rising_and_falling_rows():
    """Every chunk's logits pass all before them, or none does."""
    for vocab in (8192, 40001):
        up = torch.arange(vocab).float() / 64
        for row in (up, up.flip(0)):
            got = S.sched_beam_select(row[None].cuda(), torch.zeros(1).cuda(), 1, 128)
            want = row.topk(128).indices
            assert torch.equal(got[2].cpu(), want)


def test_rows_a_stride_apart():
    g = gen(31)
    for vocab in (100, 3001):
        x = randn(g, 6, vocab + 13, dtype=torch.bfloat16).cuda()
        s = (-torch.rand(6, generator=g)).cuda()
        a = S.sched_beam_select(x[:, 5:5 + vocab], s, 3, 3)
        b = S.sched_beam_select(x[:, 5:5 + vocab].contiguous(), s, 3, 3)
        for u, v in zip(a, b):
            assert torch.equal(u, v)


@pytest.mark.parametrize("dtype,row", [(torch.bfloat16, (4, 16)), (torch.float32, (3,)), (torch.float16, (5,)),
                                       (torch.uint8, (7,)), (torch.float32, (2,)), (torch.bfloat16, ())])
@pytest.mark.parametrize("groups,beams,outer,rows", [(1, 1, 1, 3), (2, 2, 3, 1), (3, 5, 2, 40), (2, 16, 1, 300),
                                                     (1, 128, 2, 9)])
def test_beam_reorder(dtype, row, groups, beams, outer, rows):
    g = gen(groups * 100 + beams + rows)
    n = groups * beams
    whole = (torch.randn((outer, n, rows, *row), generator=g) * 50).to(dtype)
    parents = torch.randint(0, beams, (n,), generator=g) + torch.arange(n) // beams * beams
    turned = (torch.arange(n) + 1) % beams + torch.arange(n) // beams * beams  # one cycle
    wrong = parents.clone()
    wrong[::3] = -1
    wrong[1::5] = (wrong[1::5] + beams) % (n + 7)  # of other groups, or none
    lengths = torch.randint(-1, rows + 3, (n,), generator=g)
    for p in (parents, turned, wrong, torch.arange(n)):
        for count in (None, lengths):
            got = whole.cuda()
            S.sched_beam_reorder(got, p.int().cuda(), beams, None if count is None else count.int().cuda())
            assert torch.equal(got.cpu(), R.reordered(whole, p, beams, count))


def test_reorder_of_slices():
    """Tensors inside larger ones: what lies between their rows stays."""
    g = gen(77)
    whole = randn(g, 3, 2, 8, 20, 4, 24, dtype=torch.bfloat16)
    parents = torch.randint(0, 4, (8,), generator=g) + torch.arange(8) // 4 * 4
    d = whole.cuda()
    view = d[:, 1, :, 3:15, 1]  # outer 3, slots 8, rows 12, a row of 24
    S.sched_beam_reorder(view, parents.int().cuda(), 4)
    want = whole.clone()
    want[:, 1, :, 3:15, 1] = R.reordered(whole[:, 1, :, 3:15, 1], parents, 4, None)
    assert torch.equal(d.cpu(), want)


def test_beams_keep_their_states():
    """Steps of a search: each beam's state is its tokens so far."""
    g = gen(55)
    groups, beams, vocab, steps = 3, 6, 11, 9
    for stay in (False, True):
        states = torch.full((2, groups * beams, steps), -1, dtype=torch.int32, device="cuda")
        scores = torch.full((groups * beams,), -math.inf)
        scores[::beams] = 0.0
        scores, last = scores.cuda(), None
        paths = {g * beams: [] for g in range(groups)}
        lengths = torch.zeros(groups * beams, dtype=torch.int32, device="cuda")
        for i in range(steps):
            logits = randn(g, groups * beams, vocab).cuda()
            scores, parents, last = S.sched_beam_select(logits, scores, beams, last=last, end_token=0, stay=stay)
            S.sched_beam_reorder(states, parents, beams, lengths)
            states[:, :, i] = last.int()
            lengths += 1
            paths = {s: paths[p] + [t] for s, (p, t) in enumerate(zip(parents.tolist(), last.tolist())) if p >= 0}
            for s, path in paths.items():
                assert states[0, s, :i + 1].tolist() == states[1, s, :i + 1].tolist() == path


# --- shared prefixes -----------------------------------------------------------

HALVES = [torch.float16, torch.bfloat16]


def offsets(lengths):
    at = [0]
    for x in lengths:
        at.append(at[-1] + x)
    return at


def check_shared(g, dtype, hq, hk, dim, prefixes, samples, queries, keys=None, slots=None, p_slots=None,
                 causal=True, scale=None, grad=True, size=1.0):
    """prefixes: lengths of the groups' prefixes; samples: sequences of each
    group; queries and keys: of each sequence; slots: rows that caches own."""
    keys = queries if keys is None else keys
    own_rows, pre_rows = slots or keys, p_slots or prefixes
    q_off, k_off, p_off, groups = (offsets(x) for x in (queries, own_rows, pre_rows, samples))
    q = randn(g, q_off[-1], hq, dim, dtype=dtype) * size
    k, v = randn(g, k_off[-1], hk, dim, dtype=dtype), randn(g, k_off[-1], hk, dim, dtype=dtype)
    pk, pv = randn(g, p_off[-1], hk, dim, dtype=dtype), randn(g, p_off[-1], hk, dim, dtype=dtype)
    for x, off, used in ((k, k_off, keys), (v, k_off, keys), (pk, p_off, prefixes), (pv, p_off, prefixes)):
        for a, b, n in zip(off, off[1:], used):  # behind a length: anything
            x[a + n:b] = math.nan if x is k or x is pk else math.inf
    do = randn(g, q_off[-1], hq, dim, dtype=dtype)
    k_len, p_len = keys if slots else None, prefixes if p_slots else None
    want = R.Shared(q, k, v, pk, pv, q_off, k_off, p_off, groups, k_len, p_len, causal,
                    1 / math.sqrt(dim) if scale is None else scale, do if grad else None)
    args = [x.cuda() for x in (q, k, v, pk, pv)]
    where = [i32(x) for x in (q_off, k_off, p_off, groups)]
    how = dict(k_lengths=None if k_len is None else i32(k_len), causal=causal, scale=scale,
               prefix_lengths=None if p_len is None else i32(p_len))
    out, lse = S.sched_shared_attention(*args, *where, **how)
    close(out, want.out, want.out_b, "out")
    close(lse, want.lse, want.lse_b, "lse")
    if not grad:
        return
    got = S.sched_shared_attention_grad(*args, out, lse, do.cuda(), *where, **how)
    for x, name in zip(got, ("dq", "dk", "dv", "dpk", "dpv")):
        close(x, getattr(want, name), getattr(want, name + "_b"), name)
    again = S.sched_shared_attention_grad(*args, out, lse, do.cuda(), *where, **how)
    for a, b in zip(got, again):
        assert torch.equal(a, b)  # one order of sums


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("hq,hk,dim", [(1, 1, 8), (4, 2, 32), (3, 3, 40), (8, 1, 64), (6, 2, 80), (8, 8, 128), (5, 1, 120)])
def test_shared_attention(dtype, hq, hk, dim):
    g = gen(hq * 100 + dim)
    check_shared(g, dtype, hq, hk, dim, [1], [1], [1])
    check_shared(g, dtype, hq, hk, dim, [70, 3, 129], [2, 3, 1], [14, 14, 1, 40, 2, 33])
    check_shared(g, dtype, hq, hk, dim, [64, 5], [4, 2], [3, 0, 65, 1, 64, 130], causal=False)


@pytest.mark.parametrize("dtype", HALVES)
def test_groups_sequences_and_prefixes_without_rows(dtype):
    g = gen(17)
    check_shared(g, dtype, 4, 2, 64, [0, 9, 0, 40, 5], [2, 0, 1, 3, 0], [5, 0, 3, 0, 0, 20])
    check_shared(g, dtype, 2, 2, 32, [0], [3], [0, 0, 4])
    check_shared(g, dtype, 2, 2, 32, [30, 0], [0, 2], [0, 0])
    # Own keys fewer or more than queries: rows that see the prefix alone, or nothing.
    check_shared(g, dtype, 4, 1, 64, [9, 0], [2, 3], [5, 70, 6, 7, 3], [0, 3, 9, 2, 80])
    check_shared(g, dtype, 4, 1, 64, [9, 0], [2, 3], [5, 70, 6, 7, 3], [0, 3, 0, 2, 80], causal=False)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("prefixes", [[63], [64], [65], [127, 128], [300]])
def test_prefixes_that_end_around_a_tile(dtype, prefixes):
    g = gen(prefixes[0])
    n = len(prefixes)
    check_shared(g, dtype, 4, 2, 64, prefixes, [5] * n, [13, 1, 64, 50, 0] * n)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("hq,hk,dim", [(2, 1, 32), (8, 2, 64), (32, 8, 128), (16, 1, 128)])
def test_single_tokens_over_caches(dtype, hq, hk, dim):
    g = gen(hq + dim)
    for samples in ([1], [3, 1], [20, 0, 9], [70]):
        n = sum(samples)
        keys = [(7 * i * i + 3) % 150 for i in range(n)]
        keys[0] = 0
        prefixes = [(501 * i + 77) % 900 for i in range(len(samples))]
        check_shared(g, dtype, hq, hk, dim, prefixes, samples, [1] * n, keys, slots=[150] * n,
                     p_slots=[900] * len(samples), grad=False)


@pytest.mark.parametrize("dtype", HALVES)
def test_shares_of_long_keys(dtype):
    """Prefixes and own keys that several blocks share, and their backward pass."""
    g = gen(91)
    check_shared(g, dtype, 4, 2, 64, [3000, 1111], [2, 2], [1, 2, 1, 3], [900, 1500, 1, 700], slots=[1500] * 4)
    check_shared(g, dtype, 2, 1, 128, [5000], [3], [20, 1, 33])
    check_shared(g, dtype, 8, 1, 64, [700], [2], [300, 200])


def test_tokens_behind_a_cache():
    """Some new tokens of each sequence, more than a wave's rows, over slots."""
    g = gen(14)
    check_shared(g, torch.bfloat16, 8, 2, 64, [40, 90, 7], [9, 4, 8], [40] * 21,
                 [40 + 11 * i % 70 for i in range(21)], slots=[111] * 21, p_slots=[100, 90, 64])


def test_many_short_sequences_and_many_empty_ones():
    g = gen(41)
    queries = [i % 3 for i in range(300)]
    check_shared(g, torch.bfloat16, 4, 2, 32, [21, 40], [180, 120], queries)
    queries = [0] * 170
    queries[3], queries[101], queries[169] = 5, 9, 2
    check_shared(g, torch.float16, 4, 2, 32, [21, 40], [100, 70], queries)
    check_shared(g, torch.bfloat16, 2, 2, 32, [11] * 90, [1] * 90, [i % 4 for i in range(90)])


def test_scores_of_any_size():
    g = gen(19)
    check_shared(g, torch.bfloat16, 4, 2, 64, [100], [4], [30, 20, 7, 60], size=12.0)
    check_shared(g, torch.float16, 4, 2, 64, [100], [4], [30, 20, 7, 60], scale=1.0)
    check_shared(g, torch.float16, 2, 2, 64, [100], [2], [30, 20], scale=1e-4)


@pytest.mark.parametrize("dtype", HALVES)
def test_a_shared_prefix_is_a_repeated_one(dtype):
    """Against sched_attention of sequences that each hold the prefix: out within
    two roundings; a prefix key's gradient is the sum over its copies."""
    g = gen(66)
    p, n, m, hq, hk, dim = 200, 6, 31, 8, 2, 64
    x = randn(g, n * m, hq + 2 * hk, dim, dtype=dtype).cuda()
    pre = randn(g, p, 2 * hk, dim, dtype=dtype).cuda()
    do = randn(g, n * m, hq, dim, dtype=dtype).cuda()
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    q_off, p_off, groups = i32(offsets([m] * n)), i32([0, p]), i32([0, n])
    args = (q, k, v, pre[:, :hk], pre[:, hk:])
    out, lse = S.sched_shared_attention(*args, q_off, q_off, p_off, groups)
    got = S.sched_shared_attention_grad(*args, out, lse, do, q_off, q_off, p_off, groups)
    whole = torch.cat([torch.cat([pre, x[i * m:(i + 1) * m, hq:]]) for i in range(n)])
    k_off = i32(offsets([p + m] * n))
    out2, lse2 = S.sched_attention(q, whole[:, :hk], whole[:, hk:], q_off, k_off)
    d = S.sched_attention_grad(q, whole[:, :hk], whole[:, hk:], out2, lse2, do, q_off, k_off)
    u = R.U[dtype]
    for a, b in ((out, out2), (got[0], d[0])):
        assert float((a.double() - b.double()).norm() / b.double().norm()) < 2 * u
    for a, b in ((got[3], d[1]), (got[4], d[2])):
        b = b.double().view(n, p + m, hk, dim)[:, :p].sum(0)
        assert float((a.double() - b).norm() / b.norm()) < 2 * u
    for a, b in ((got[1], d[1]), (got[2], d[2])):
        b = b.double().view(n, p + m, hk, dim)[:, p:].reshape(n * m, hk, dim)
        assert float((a.double() - b).norm() / b.norm()) < 2 * u


def test_rows_outside_the_groups_stay():
    """Rows behind the last sequence and prefix, on both paths."""
    g = gen(23)
    for lengths, queries in ((None, [3, 5, 4]), ([1, 9, 6], [1, 1, 1])):
        keys = [9, 9, 9] if lengths else queries
        q_off, k_off, p_off, groups = offsets(queries), offsets(keys), [0, 20, 33], [0, 2, 3]
        q = randn(g, q_off[-1] + 7, 4, 32, dtype=torch.bfloat16).cuda()
        k, v = (randn(g, k_off[-1] + 70, 2, 32, dtype=torch.bfloat16).cuda() for _ in range(2))
        pk, pv = (randn(g, 33 + 90, 2, 32, dtype=torch.bfloat16).cuda() for _ in range(2))
        where = [i32(x) for x in (q_off, k_off, p_off, groups)]
        n = None if lengths is None else i32(lengths)
        out, lse = torch.full_like(q, 7), torch.full((4, q.shape[0]), 7.0, device="cuda")
        S.sched_shared_attention(q, k, v, pk, pv, *where, k_lengths=n, out=out, lse=lse)
        assert bool((out[q_off[-1]:] == 7).all()) and bool((lse[:, q_off[-1]:] == 7).all())
        assert not bool((out[:q_off[-1]] == 7).all(2).any())
        grads = [torch.full_like(x, 7) for x in (q, k, v, pk, pv)]
        S.sched_shared_attention_grad(q, k, v, pk, pv, out, lse, q, *where, k_lengths=n, d_q=grads[0],
                                      d_k=grads[1], d_v=grads[2], d_prefix_k=grads[3], d_prefix_v=grads[4])
        for x, end in zip(grads, (q_off[-1], k_off[-1], k_off[-1], 33, 33)):
            assert bool((x[end:] == 7).all()) and not bool((x[:end] == 7).all(2).any())


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_no_number_stays_in_its_sequence(dtype, bad):
    """A sequence whose tensors hold NaN or infinities leaves the others of its
    tile as they are; they share the prefix, whose gradient it reaches."""
    g = gen(37)
    queries = [14, 9, 20, 14, 3, 30]
    off, p_off, groups, hq, hk, dim = offsets(queries), [0, 71, 90], [0, 4, 6], 4, 2, 64
    x = [randn(g, off[-1], h, dim, dtype=dtype) for h in (hq, hk, hk, hq)]
    pre = [randn(g, 90, hk, dim, dtype=dtype) for _ in range(2)]
    where = [i32(t) for t in (off, off, p_off, groups)]
    want = R.Shared(*x[:3], *pre, off, off, p_off, groups, None, None, True, 0.125, x[3])
    keep = torch.ones(off[-1], dtype=torch.bool)
    keep[off[1]:off[2]] = False
    for i in range(4):
        spoiled = [t.clone() for t in x]
        spoiled[i][off[1] + 4, 0, 3] = bad
        q, k, v, pk, pv, do = (t.cuda() for t in (*spoiled[:3], *pre, spoiled[3]))
        out, lse = S.sched_shared_attention(q, k, v, pk, pv, *where)
        got = out, lse.t(), *S.sched_shared_attention_grad(q, k, v, pk, pv, out, lse, do, *where)
        for a, name in zip(got, ("out", "lse", "dq", "dk", "dv")):
            b, bound = getattr(want, name), getattr(want, name + "_b")
            b, bound = (t.t() if name == "lse" else t for t in (b, bound))
            close(a[keep.cuda()], b[keep], bound[keep], (i, name))
        shows = got[0] if i < 3 else got[2]
        assert not bool(torch.isfinite(shows[off[1]:off[2]].float()).all())
        for a, name in zip(got[5:], ("dpk", "dpv")):  # the other group's prefix
            close(a[71:], getattr(want, name)[71:], getattr(want, name + "_b")[71:], (i, name))


def test_shared_attention_grad_against_differences():
    """Along random directions, in 64 bits, at a size that bf16 holds exactly."""
    g = gen(5)
    q_off, p_off, groups, do = [0, 6, 10], [0, 9], [0, 2], randn(g, 10, 2, 16, dtype=torch.bfloat16)
    x = [randn(g, n, h, 16, dtype=torch.bfloat16) for n, h in ((10, 2), (10, 1), (10, 1), (9, 1), (9, 1))]
    step = [randn(g, *t.shape) for t in x]
    d = [t.cuda() for t in x]
    where = [i32(t) for t in (q_off, q_off, p_off, groups)]
    out, lse = S.sched_shared_attention(*d, *where)
    got = S.sched_shared_attention_grad(*d, out, lse, do.cuda(), *where)

    def loss(h):
        y = [t.double() + h * s for t, s in zip(x, step)]
        total = 0.0
        for b in range(2):
            r = slice(q_off[b], q_off[b + 1])
            m = r.stop - r.start
            for head in range(2):
                k, v = torch.cat([y[3][:, 0], y[1][r, 0]]), torch.cat([y[4][:, 0], y[2][r, 0]])
                a = y[0][r, head] @ k.T * R.f32(0.25)
                a[:, 9:][torch.arange(m)[None] > torch.arange(m)[:, None]] = -math.inf
                total += float((torch.softmax(a, 1) @ v * do[r, head].double()).sum())
        return total

    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    parts = [(a.cpu().double() * s).sum() for a, s in zip(got, step)]
    size = math.sqrt(sum(float((a.cpu().double() * s).square().sum()) for a, s in zip(got, step)))
    # Every gradient is off by up to three roundings of 2^-8 of itself and of what
    # cancels in it (of the same size), with random signs: 4 sigma of it.
    assert abs(slope - float(sum(parts))) < 4 * 3 * 2.0 ** -8 * size


# --- streams, graphs, workspaces -------------------------------------------------


def beam_step(logits, scores, states, **kw):
    out = S.sched_beam_select(logits, scores, 4, 4, stay=True, **kw)
    S.sched_beam_reorder(states, out[1], 4, stream=kw.get("stream"))
    return out


def test_on_another_stream():
    g = gen(2)
    logits, scores = randn(g, 8, 9001).cuda(), (-torch.rand(8, generator=g)).cuda()
    states = randn(g, 2, 8, 30, 16).cuda()
    x, p, f = randn(g, 50, 4, 32).cuda(), torch.arange(50, device="cuda"), torch.rand(16, generator=g).cuda()
    h = randn(g, 40, 4, 32, dtype=torch.bfloat16).cuda()
    where = [i32(t) for t in ([0, 20, 40], [0, 20, 40], [0, 40], [0, 2])]

    def attend(**kw):
        out, lse = S.sched_shared_attention(h, h, h, h, h, *where, **kw)
        return (out, lse, *S.sched_shared_attention_grad(h, h, h, h, h, out, lse, h, *where, **kw))

    here = states.clone()
    want = beam_step(logits, scores, here), S.sched_norm_rotate(x, x, p, f), attend()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    there = states.clone()
    stream.wait_stream(torch.cuda.current_stream())
    got = (beam_step(logits, scores, there, stream=stream), S.sched_norm_rotate(x, x, p, f, stream=stream),
           attend(stream=stream))
    torch.cuda.current_stream().wait_stream(stream)
    for a, b in zip((*want[0], *want[1], *want[2], here), (*got[0], *got[1], *got[2], there)):
        assert torch.equal(a, b)


def test_captured_in_a_graph():
    """A step of the search and a turned projection, replayed on new inputs."""
    g = gen(21)
    draws = [(randn(g, 8, 5001).cuda(), (-torch.rand(8, generator=g)).cuda(), randn(g, 2, 8, 30, 16).cuda(),
              randn(g, 20, 6, 32).cuda()) for _ in range(4)]
    logits, scores, states, x = (t.clone() for t in draws[0])
    pos, f, w = torch.arange(20, device="cuda"), torch.rand(16, generator=g).cuda(), torch.ones(32, device="cuda")
    where = [i32(t) for t in ([0, 8, 20], [0, 8, 20], [0, 20], [0, 2])]
    lengths = i32([8, 5])

    def run(logits, scores, states, x):
        out = beam_step(logits, scores, states)
        q, k = S.sched_norm_rotate(x[:, :4], x[:, 4:], pos, f, w, w)
        h, v = x[:, 4:].bfloat16(), q.bfloat16()
        attended = []
        for n in (None, lengths):  # packed, and single tokens' way
            o, lse = S.sched_shared_attention(v, h, h, h, h, *where, k_lengths=n)
            attended += [o, lse, *S.sched_shared_attention_grad(v, h, h, h, h, o, lse, v, *where, k_lengths=n)]
        return (*out, q, k, *attended, *S.sched_norm_rotate_grad(x[:, :4], x[:, 4:], q, k, pos, f, w, w))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(logits, scores, states, x)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(logits, scores, states, x)
    for draw in draws[1:] + draws:
        for a, b in zip((logits, scores, states, x), draw):
            a.copy_(b)
        graph.replay()
        eager = [t.clone() for t in draw]
        want = run(*eager)
        torch.cuda.synchronize()
        for a, b in zip((*got, states), (*want, eager[2])):
            assert torch.equal(a, b)


# --- far rows ------------------------------------------------------------------


@pytest.mark.parametrize("step", [(1 << 23) + 8, (1 << 24) + 8])
def test_rows_far_apart(step):
    """Offsets that pass 32 bits, at distances that a tile's lanes can add up and at
    others: the same bits as rows next to each other."""
    g = gen(30)
    dim, kv, rows = 64, 2, 264
    whole = torch.empty((rows - 1) * step + 2 * kv * dim, dtype=torch.bfloat16, device="cuda")
    far = whole.as_strided((rows, 2 * kv, dim), (step, dim, 1))
    near = randn(g, rows, 2 * kv, dim, dtype=torch.bfloat16).cuda()
    far.copy_(near)
    q = randn(g, 60, 4, dim, dtype=torch.bfloat16).cuda()

    def run(x, grads, **kw):
        pre, own = x[:200], x[200:]
        where = [i32(t) for t in ([0, 25, 60], [0, 30, 64], [0, 200], [0, 2])]
        args = (q, own[:, :kv], own[:, kv:], pre[:, :kv], pre[:, kv:])
        out, lse = S.sched_shared_attention(*args, *where, **kw)
        to = {} if grads is None else dict(d_k=grads[200:, :kv], d_v=grads[200:, kv:],
                                           d_prefix_k=grads[:200, :kv], d_prefix_v=grads[:200, kv:])
        return out, lse, *S.sched_shared_attention_grad(*args, out, lse, q, *where, **kw, **to)

    for lengths in (None, i32([30, 17])):
        want = run(near, None, k_lengths=lengths)
        for a, b in zip(want, run(far, None, k_lengths=lengths)):
            assert torch.equal(a, b)
    far.zero_()
    got = run(near, far)
    for a, b in zip(run(near, None), got):
        assert torch.equal(a, b)
    # Rows of a cache as far apart, and the gradient from there.
    pos, freq = torch.arange(rows, device="cuda"), torch.rand(32, generator=g).cuda()
    places = torch.randperm(rows, generator=g).cuda()
    k, v = near[:, :kv], near[:, kv:]
    a = S.sched_norm_rotate(k, k, pos, freq, v=v)
    b = S.sched_norm_rotate(k, k, pos, freq, v=v, places=places, k_out=far[:, :kv], v_out=far[:, kv:])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1][places]) and torch.equal(a[2], b[2][places])
    a = S.sched_norm_rotate_grad(k, k, k, far[:, :kv][places], pos, freq)
    b = S.sched_norm_rotate_grad(k, k, k, far[:, :kv], pos, freq, places=places)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_states_of_more_than_4_gib():
    n = (1 << 30) + 24  # of 4 bytes
    x = torch.arange(n, dtype=torch.int32, device="cuda")
    states = torch.stack([x, x * 3, x * 5]).view(1, 3, 8, -1)
    S.sched_beam_reorder(states, i32([2, 0, 1]), 3)
    for i, f in enumerate((5, 1, 3)):
        assert torch.equal(states[0, i].view(-1), x * f)


def test_beam_select_of_the_longest_rows():
    g = gen(31)
    vocab = 1 << 22
    logits, scores = torch.randn((3, vocab), generator=g).cuda() * 3, torch.tensor([-1.0, -2.0, -1.5]).cuda()
    logits[0, -1], logits[1, -1] = 19.0, 21.0
    z = torch.log_softmax(logits.double(), 1) + scores.double()[:, None]
    best = z.view(-1).topk(7)
    assert float((best.values[:-1] - best.values[1:]).min()) > 1e-5
    got = S.sched_beam_select(logits, scores, 3, 6)
    assert torch.equal(got[1].long(), best.indices[:-1] // vocab)
    assert torch.equal(got[2], best.indices[:-1] % vocab)


def test_calls_at_once():
    """The same calls on two streams at a time, with workspaces of their own."""
    g = gen(32)
    logits = [randn(g, 16, 30011).cuda() for _ in range(2)]
    scores = torch.zeros(16, device="cuda")
    h = [randn(g, 900, 4, 64, dtype=torch.bfloat16).cuda() for _ in range(2)]
    where = [i32(t) for t in ([0, 400, 900], [0, 400, 900], [0, 900], [0, 2])]

    def run(i, **kw):
        a = (h[i],) * 5
        out, lse = S.sched_shared_attention(*a, *where, **kw)
        return (*S.sched_beam_select(logits[i], scores, 8, **kw), out, lse,
                *S.sched_shared_attention_grad(*a, out, lse, h[i], *where, **kw))

    want = [run(0), run(1)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[run(i, stream=streams[i]) for i in range(2)] for _ in range(3)]
    torch.cuda.synchronize()
    for pair in got:
        for a, b in zip(pair, want):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


def test_numbers_that_no_type_holds():
    x, s, h = torch.zeros((4, 9), device="cuda"), torch.zeros(4, device="cuda"), torch.zeros((4, 2, 8), device="cuda")
    at = torch.arange(4, device="cuda")
    for call in (lambda: S.sched_beam_select(x, s, 2, end_token=1 << 70), lambda: S.sched_beam_select(x, s, 2, 1 << 40),
                 lambda: S.sched_beam_select(x, s, 2, temperature=1e300), lambda: S.sched_norm_rotate(h, h, at, None, eps=1e39),
                 lambda: S.sched_norm_rotate(h, h, at, None, norm=1 << 32),
                 lambda: S.sched_beam_reorder(h[None], at.int(), (1 << 32) + 2)):
        with pytest.raises(S.SchedError):
            call()
    b = h.bfloat16()
    with pytest.raises(S.SchedError):
        S.sched_attention(b, b, b, i32([0, 4]), i32([0, 4]), scale=1e300)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("hq,hk,dim,prefixes,samples,lo,hi", [(32, 4, 16, [1, 2, 2, 1], 3, 6, 31), (8, 2, 64, [40, 9], 5, 1, 20),
                                                             (4, 1, 128, [30], 8, 14, 14)])
def test_small_calls_are_rounded_once(dtype, hq, hk, dim, prefixes, samples, lo, hi):
    """Of rows that see up to 64 keys.  Probabilities and dS are known to 2^-16 of
    themselves or better and all else to 2^-20, where a result's rounding is 2^-9 or
    2^-12 of it: in norm nothing beside it."""
    g = gen(dim)
    lengths = torch.randint(lo, hi + 1, (len(prefixes) * samples,), generator=g).tolist()
    off, p_off, groups = offsets(lengths), offsets(prefixes), offsets([samples] * len(prefixes))
    q, do = (randn(g, off[-1], hq, dim, dtype=dtype) for _ in range(2))
    k, v = (randn(g, off[-1], hk, dim, dtype=dtype) for _ in range(2))
    pk, pv = (randn(g, p_off[-1], hk, dim, dtype=dtype) for _ in range(2))
    want = R.Shared(q, k, v, pk, pv, off, off, p_off, groups, None, None, True, 1 / math.sqrt(dim), do)
    args, where = [x.cuda() for x in (q, k, v, pk, pv)], [i32(x) for x in (off, off, p_off, groups)]
    out, lse = S.sched_shared_attention(*args, *where)
    grads = S.sched_shared_attention_grad(*args, out, lse, do.cuda(), *where)
    for x, name in zip((out, *grads), ("out", "dq", "dk", "dv", "dpk", "dpv")):
        y = getattr(want, name)
        once = float((y.to(dtype).double() - y).norm())
        assert float((x.cpu().double() - y).norm()) < 1.1 * once, name


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("hq,hk,dim", [(8, 2, 64), (8, 1, 128), (9, 3, 120)])
def test_calls_that_are_not_small(dtype, hq, hk, dim):
    """More than 2^21 pairs of a row and a key: products of rounded operands alone."""
    g = gen(hq + dim)
    check_shared(g, dtype, hq, hk, dim, [400, 333], [3, 3], [100, 130, 77, 120, 99, 110])
    check_shared(g, dtype, hq, hk, dim, [900], [5], [70, 0, 64, 129, 1], [100, 20, 64, 200, 30],
                 slots=[200] * 5, p_slots=[1000], causal=False)
    check_shared(g, dtype, 32, 8, dim, [1500, 1300], [20, 35], [1] * 55, [(31 * i) % 400 for i in range(55)],
                 slots=[400] * 55, p_slots=[1600] * 2, grad=False)
    # Of few rows to a sequence, of short prefixes, and of few keys.
    check_shared(g, dtype, 16, 8, dim, [1000], [100], [1, 2] * 50)
    check_shared(g, dtype, 8, 2, dim, [40], [6], [200] * 6)
    check_shared(g, dtype, 16, 4, dim, [90], [60], [20] * 60)


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_no_number_stays_in_its_sequence_of_larger_calls(dtype, bad):
    g = gen(38)
    queries = [(5 * i) % 31 for i in range(40)]
    off, p_off, groups, hq, hk, dim = offsets(queries), [0, 700, 1120], [0, 25, 40], 16, 8, 64
    x = [randn(g, off[-1], h, dim, dtype=dtype) for h in (hq, hk, hk, hq)]
    pre = [randn(g, 1120, hk, dim, dtype=dtype) for _ in range(2)]
    where = [i32(t) for t in (off, off, p_off, groups)]
    want = R.Shared(*x[:3], *pre, off, off, p_off, groups, None, None, True, 0.125, x[3])
    keep = torch.ones(off[-1], dtype=torch.bool)
    keep[off[11]:off[12]] = False
    for i in range(4):
        spoiled = [t.clone() for t in x]
        spoiled[i][off[11] + 4, 0, 3] = bad
        q, k, v, pk, pv, do = (t.cuda() for t in (*spoiled[:3], *pre, spoiled[3]))
        out, lse = S.sched_shared_attention(q, k, v, pk, pv, *where)
        got = out, lse.t(), *S.sched_shared_attention_grad(q, k, v, pk, pv, out, lse, do, *where)
        for a, name in zip(got, ("out", "lse", "dq", "dk", "dv")):
            b, bound = getattr(want, name), getattr(want, name + "_b")
            b, bound = (t.t() if name == "lse" else t for t in (b, bound))
            close(a[keep.cuda()], b[keep], bound[keep], (i, name))
        for a, name in zip(got[5:], ("dpk", "dpv")):  # the other group's prefix
            close(a[700:], getattr(want, name)[700:], getattr(want, name + "_b")[700:], (i, name))


def test_beam_select_of_many_groups_and_of_short_strips():
    check_beams(gen(60), 300, 4, 4, 20, torch.float32, stay=True)
    check_beams(gen(61), 300, 2, 2, 700, torch.float32)
    check_beams(gen(62), 2, 40, 40, 6300, torch.float32, stay=True)
    check_beams(gen(63), 3, 5, 100, 300, torch.float32)
    check_beams(gen(64), 1, 2, 128, 1500, torch.float32)
    check_beams(gen(65), 2, 16, 16, 64, torch.float32)
