"""The operators that serve many answers to one prompt, at the ends of their
ranges: logits far from zero, what is no number beside what is."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from answers64 import Shared, beam_results  # noqa: E402
from policy64 import F, close, f32  # noqa: E402
from test_gpu_answers import check_shared, i32, offsets  # noqa: E402

import paper_2607_22242_amd as S  # noqa: E402

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype)


# --- beams far from zero ---------------------------------------------------------


def candidates(logits, scores, beams, temperature):
    """Per group a list of (score, beam, token), best first, equal ones by beam and
    token.  A row's greatest logit is taken away first, so that what all logits of a
    row have in common never meets the score; a greatest logit that is not finite
    leaves no candidate."""
    groups = [[] for _ in range(logits.shape[0] // beams)]
    for i, row in enumerate(logits.double()):
        start, most = float(scores[i]), float(row.max())
        if not math.isfinite(start) or not math.isfinite(most):
            continue
        z = (row - most) / f32(temperature)
        base = start - math.log(float(torch.exp(z).sum()))
        groups[i // beams] += [(base + x, i % beams, t) for t, x in enumerate(z.tolist()) if x > -math.inf]
    for found in groups:
        found.sort(key=lambda c: (-c[0], c[1], c[2]))
    return groups


def check_far_beams(logits, scores, beams, width, temperature, stay=False):
    groups = candidates(logits, scores, beams, temperature)
    for found in groups:
        # Beams that 64-bit scores tell apart by a lot, whatever the sums' errors.
        for a, b in zip(found[:width], found[1:width + 1]):
            assert a[1] == b[1] or a[0] == b[0] or a[0] - b[0] > 1e-4 + 1e-12 * abs(a[0]), "input"
    want = beam_results(groups, beams, width, stay)
    got = S.sched_beam_select(logits.cuda(), scores.cuda(), beams, width, temperature=temperature, stay=stay)
    assert torch.equal(got[1].cpu().long(), want[1]), "parents"
    assert torch.equal(got[2].cpu(), want[2]), "tokens"
    # A power with exponent -a is off by 2^-24 (2 a + 2) of itself, and the powers' sum
    # of a's by less than log2(n) of theirs; a lane adds n / 64 of them and the
    # reference moves; the result is rounded.  Nothing grows with what a row's logits
    # have in common.
    n = logits.shape[1]
    close(got[0], want[0], F * (16 * math.log2(n + 1) + n / 64 + 64 + want[0].nan_to_num(0, 0, 0).abs()), "scores")


FAR_ROWS = [3, 256, 700, 5003]  # a group's own reading of logits, and strips of rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", FAR_ROWS)
def test_beams_of_the_lowest_logits(dtype, vocab):
    """A row whose tokens are all masked with the type's lowest number has equal
    log-probabilities, not the best ones."""
    beams = 4
    logits = (randn(gen(vocab), 2 * beams, vocab) * 2).to(dtype)
    scores = torch.linspace(-4, -4.5, 2 * beams)
    logits[1] = torch.finfo(dtype).min       # among ordinary beams
    logits[beams:] = torch.finfo(dtype).min  # a group of such rows
    logits[beams + 2, vocab // 2] = 1.0      # and one with a single token left
    for stay in (False, True):
        check_far_beams(logits, scores, beams, beams, 1.0, stay)


@pytest.mark.parametrize("dtype,offset", [(torch.float32, 1e20), (torch.float32, -1e20), (torch.float32, 3e38),
                                          (torch.bfloat16, 1e20), (torch.bfloat16, -3e38), (torch.float16, 6e4)])
@pytest.mark.parametrize("vocab", FAR_ROWS)
def test_beams_of_rows_with_an_offset(dtype, offset, vocab):
    """Logits whose steps, at that distance from zero, are far more than 1, and one value
    all over: scores are what the beams had, less the logarithm of how many there are."""
    g = gen(vocab + 1)
    beams = 5
    logits = torch.full((beams, vocab), offset).to(dtype)
    logits[0] = randn(g, vocab).to(dtype)
    up = torch.rand((2, vocab), generator=g) < 0.3  # a step or two above it
    logits[2:4] = torch.where(up, logits[2:4] * (1 + 4 * torch.finfo(dtype).eps), logits[2:4]).to(dtype)
    logits[2:4][torch.isinf(logits[2:4])] = offset
    scores = torch.tensor([-6.0, -5.0, -4.5, -5.7, -3.9])
    check_far_beams(logits, scores, beams, beams, 1.0)
    check_far_beams(logits, scores, beams, beams, 0.7, stay=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("temperature", [1e-12, 1e-20, 1e-30])
@pytest.mark.parametrize("vocab", FAR_ROWS)
def test_beams_at_the_lowest_temperatures(dtype, temperature, vocab):
    """Every beam's best token goes on with the score that the beam had."""
    beams = 6
    logits = randn(gen(vocab + 2), beams, vocab).to(dtype)
    logits[:, vocab // 3] = torch.arange(beams).to(dtype) + 8
    scores = torch.tensor([-6.0, -5.0, -4.5, -5.7, -3.9, -4.1])
    check_far_beams(logits, scores, beams, beams, temperature)
    check_far_beams(logits, scores, beams, beams, temperature, stay=True)


# --- shared prefixes of very unequal lengths -----------------------------------------

HALVES = [torch.float16, torch.bfloat16]


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("prefixes", [[4000, 10], [3000, 0], [10, 5000]])
def test_short_answers_behind_unequal_prefixes(dtype, prefixes):
    """Blocks share the long prefix' keys, and the other group's rows see a tile of
    keys at most."""
    check_shared(gen(prefixes[0]), dtype, 4, 2, 64, prefixes, [4, 4], [10, 9, 12, 10, 10, 1, 10, 8])
    check_shared(gen(prefixes[1]), dtype, 4, 2, 128, prefixes, [4, 4], [10] * 8, [10, 40, 0, 9, 10, 7, 30, 10],
                 slots=[40] * 8, p_slots=[5000, 5000])


@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("prefixes", [[4000, 10], [0, 4000]])
def test_what_is_no_number_stays_in_its_sequence_where_blocks_share_prefixes(dtype, bad, prefixes):
    """Each of the blocks that share a group's prefix forms its rows' delta for itself."""
    g = gen(39)
    queries, hq, hk, dim = [10, 9, 12, 10, 10, 4, 10, 8], 4, 2, 64
    off, p_off, groups = offsets(queries), offsets(prefixes), [0, 4, 8]
    short = 4 if prefixes[0] > prefixes[1] else 0  # the first sequence of the short prefix
    x = [randn(g, off[-1], h, dim, dtype=dtype) for h in (hq, hk, hk, hq)]
    pre = [randn(g, p_off[-1], hk, dim, dtype=dtype) for _ in range(2)]
    where = [i32(t) for t in (off, off, p_off, groups)]
    want = Shared(*x[:3], *pre, off, off, p_off, groups, None, None, True, 0.125, x[3])
    there = torch.arange(p_off[-1])
    for spoiled in (short + 2, (short + 5) % 8):  # of either group
        keep = torch.ones(off[-1], dtype=torch.bool)
        keep[off[spoiled]:off[spoiled + 1]] = False
        its = 0 if spoiled < 4 else 1
        others = (there < p_off[its]) | (there >= p_off[its + 1])
        for i in range(4):
            y = [t.clone() for t in x]
            y[i][off[spoiled] + 3, 0, 3] = bad
            q, k, v, pk, pv, do = (t.cuda() for t in (*y[:3], *pre, y[3]))
            out, lse = S.sched_shared_attention(q, k, v, pk, pv, *where)
            got = out, lse.t(), *S.sched_shared_attention_grad(q, k, v, pk, pv, out, lse, do, *where)
            for a, name in zip(got, ("out", "lse", "dq", "dk", "dv")):
                b, bound = getattr(want, name), getattr(want, name + "_b")
                b, bound = (t.t() if name == "lse" else t for t in (b, bound))
                close(a[keep.cuda()], b[keep], bound[keep], (spoiled, i, name))
            for a, name in zip(got[5:], ("dpk", "dpv")):  # the other group's prefix
                close(a[others.cuda()], getattr(want, name)[others], getattr(want, name + "_b")[others],
                      (spoiled, i, name))


# --- elements that are not turned -----------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved,dim,turned", [(True, 16, 6), (True, 64, 2), (True, 128, 64), (False, 64, 32),
                                                    (False, 40, 20), (True, 24, 0)])
def test_elements_that_are_not_turned_stay(dtype, interleaved, dim, turned):
    """Whatever their neighbours hold, infinities and NaN among them; what is turned
    does not meet them."""
    g = gen(dim + turned)
    x, pos = randn(g, 11, 5, dim, dtype=dtype), torch.arange(11).cuda()
    freq = torch.rand(turned // 2, generator=g).cuda() if turned else None
    how = dict(norm=False, interleaved=interleaved)
    odd = x.clone()
    for i, e in enumerate(range(turned, dim, 3)):
        odd[i % 11, i % 5, e] = (math.inf, -math.inf, math.nan)[i % 3]

    def run(t):
        t = t.cuda()
        forward = S.sched_norm_rotate(t[:, :3], t[:, 3:], pos, freq, **how)
        back = S.sched_norm_rotate_grad(t[:, :3], t[:, 3:], t[:, :3], t[:, 3:], pos, freq, **how)[:2]
        return [torch.cat(y, 1).cpu() for y in (forward, back)]

    for a, b in zip(run(x), run(odd)):
        assert torch.equal(a[..., :turned], b[..., :turned])
        for got, want in ((a, x), (b, odd)):
            got, want = got[..., turned:].float(), want[..., turned:].float()
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got, 7.0), torch.nan_to_num(want, 7.0))


# --- batches without rows -------------------------------------------------------------


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows_of_a_joint_projection(dtype):
    """Slices of a projection of no rows, with results of their own: tensors without
    memory are not the same memory."""
    hq, hk, dim = 4, 2, 32
    x = torch.empty((0, hq + 2 * hk, dim), dtype=dtype, device="cuda")
    q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    p, f = torch.empty(0, dtype=torch.int64, device="cuda"), torch.ones(dim // 2, device="cuda")
    w = torch.ones(dim, device="cuda")
    for t in S.sched_norm_rotate(q, k, p, f, w, w, v=v):
        assert t.shape[0] == 0 and t.dtype == dtype
    out = torch.empty_like(x)
    S.sched_norm_rotate(q, k, p, f, w, w, v=v, q_out=out[:, :hq], k_out=out[:, hq:hq + hk], v_out=out[:, hq + hk:])
    cache = torch.ones((2, 4, hk, dim), dtype=dtype, device="cuda")
    S.sched_norm_rotate(q, k, p, f, w, w, v=v, places=p, k_out=cache[0], v_out=cache[1])
    assert bool((cache == 1).all())
    d_q, d_k = (torch.empty((0, h, dim), dtype=dtype, device="cuda") for h in (hq, hk))
    for places, d_k_out in ((None, d_k), (p, cache[0])):
        got = S.sched_norm_rotate_grad(q, k, d_q, d_k_out, p, f, w, w, places=places)
        assert got[0].shape == (0, hq, dim) and got[1].shape == (0, hk, dim)
        assert not bool(got[2].any()) and not bool(got[3].any())
    d = torch.empty_like(x)
    S.sched_norm_rotate_grad(q, k, d_q, d_k, p, f, d_q=d[:, :hq], d_k=d[:, hq:hq + hk])
