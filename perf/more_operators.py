"""Operators of a mapping agent that answers many times to one prompt, one dict of plain values each.

The agent reads a workflow's tool cards once and gives many answers to them:
samples whose makespans it learns from, or beams of which it keeps the best.
A case is one pass through an operator of that work, the way a program calls
it: tensors on the GPU, ragged sequences packed one after the other or in slots
of a cache, int32 offsets on the device.

rotate   norms of the queries' and keys' heads and their rotation by position;
         of single tokens into a cache ("cached"), else with its gradient
answer   attention of single tokens over the group's shared prefix and the
         sequence's own cache
update   attention of packed answers over the group's shared prefix and
         themselves, and its backward pass
beams    the best continuations of each group's beams, and the beams' caches
         following them

`run` computes these in elementary torch operations in 32 bits (64 for angles,
and for scores next to the border of a selection), or by the package's
operators where `own` is true; `exact` in 64 bits, from the definitions.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # The agent answering: one new token for each of 48 sequences, its keys
        # and values to their rows of the cache; a call's latency.
        dict(name="rotate token", op="rotate", dtype="bf16", rows=48, q_heads=32, kv_heads=8, dim=128,
             turned=128, interleaved=False, cached=True, slot=100),
        # A small model's training step in 32 bits; heads of which half is
        # turned, in pairs that are no multiple of eight apart.
        dict(name="rotate cards", op="rotate", dtype="f32", rows=1001, q_heads=4, kv_heads=2, dim=40,
             turned=20, interleaved=False, cached=False, slot=0),
        # The largest: 65,536 tokens of a training step.
        dict(name="rotate 65536", op="rotate", dtype="bf16", rows=65536, q_heads=32, kv_heads=8, dim=128,
             turned=128, interleaved=False, cached=False, slot=0),
        # Four workflows, 16 answers each, prompts of tool cards, a few tokens
        # answered so far: latency.
        dict(name="answer 4x16", op="answer", dtype="f16", groups=4, samples=16, p_lo=60, p_hi=300,
             lo=1, hi=20, slot=24, q_heads=8, kv_heads=2, dim=64),
        # An ordinary round of sampling: 8 prompts of up to 6,000 tokens, 64
        # answers each, up to 400 tokens so far.
        dict(name="answer 8x64", op="answer", dtype="bf16", groups=8, samples=64, p_lo=500, p_hi=6000,
             lo=1, hi=400, slot=512, q_heads=32, kv_heads=8, dim=128),
        # Few answers to very long prompts.
        dict(name="answer long", op="answer", dtype="bf16", groups=2, samples=4, p_lo=20000,
             p_hi=32000, lo=1, hi=2000, slot=4096, q_heads=64, kv_heads=8, dim=128),
        # The agent's own update: 13 scenarios x 64 sampled mappings of 14
        # tools, prompts of five tokens a tool and a start.
        dict(name="update modes", op="update", dtype="bf16", groups=13, samples=64, p_lo=71, p_hi=71,
             lo=14, hi=14, q_heads=4, kv_heads=2, dim=32),
        # An ordinary update: reasoned answers of ragged lengths, ragged prompts.
        dict(name="update ragged", op="update", dtype="f16", groups=8, samples=8, p_lo=300, p_hi=2500,
             lo=20, hi=300, q_heads=16, kv_heads=4, dim=128),
        # The largest: 16 answers of 512 tokens to one prompt of 8,192.
        dict(name="update 8192", op="update", dtype="bf16", groups=1, samples=16, p_lo=8192, p_hi=8192,
             lo=512, hi=512, q_heads=32, kv_heads=8, dim=128),
        # Beams of mappings, a mode per tool: 13 scenarios x 64 beams, three
        # logits each, the small model's caches; results by score.
        dict(name="beams modes", op="beams", dtype="f32", vocab=3, groups=13, beams=64, width=64,
             stay=False, end=-1, outer=4, rows=14, row=64, temperature=1.0),
        # An ordinary vocabulary of odd size, some beams finished.
        dict(name="beams 32003", op="beams", dtype="bf16", vocab=32003, groups=8, beams=8, width=8,
             stay=True, end=2, outer=8, rows=300, row=512, temperature=0.7),
        # The largest: 16 groups of 16 beams, a vocabulary of 131072.
        dict(name="beams 131072", op="beams", dtype="bf16", vocab=131072, groups=16, beams=16, width=16,
             stay=True, end=-1, outer=16, rows=160, row=512, temperature=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "rotate", "answer", "answer", "update", "update", "beams", "beams"])
    if op == "rotate":
        kv = rng.choice([1, 2, 3, 4, 8])
        heads, dim = kv * rng.choice([1, 2, 3, 4, 8]), rng.choice([16, 40, 64, 80, 96, 120, 128, 128, 256])
        cached = rng.random() < 0.4
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        room = 65536 * 40 * 128 * 2 // ((heads + 2 * kv) * dim * BYTES[dtype])
        rows = min(_log(rng, 1, 700), room) if cached else min(_log(rng, 1, 65536), room)
        turned = dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
        return dict(op=op, dtype=dtype, rows=rows, q_heads=heads, kv_heads=kv, dim=dim, turned=turned,
                    interleaved=rng.random() < 0.3, cached=cached,
                    slot=rng.randint(1, 100) if cached else 0)
    if op == "beams":
        vocab, beams = _log(rng, 2, 131072), _log(rng, 1, 64)
        dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
        groups = max(1, min(_log(rng, 1, 30), 256 * 131072 * 2 // (vocab * beams * BYTES[dtype])))
        width = beams if beams > 1 else _log(rng, 1, 32)
        outer, rows = _log(rng, 1, 16), _log(rng, 1, 300)
        row = max(8, min(8 * _log(rng, 1, 128), 16 * 256 * 160 * 512 // (outer * rows * groups * width)) // 8 * 8)
        return dict(op=op, dtype=dtype, vocab=vocab, groups=groups, beams=beams, width=width,
                    stay=width == beams and rng.random() < 0.6,
                    end=rng.choice([-1, rng.randrange(vocab)]), outer=outer, rows=rows, row=row,
                    temperature=rng.choice([0.7, 1.0, 1.3]))
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 8])
    dim = rng.choice([16, 32, 40, 64, 64, 80, 96, 120, 128, 128, 128])
    dtype = rng.choice(["f16", "bf16", "bf16"])
    groups, samples = _log(rng, 1, 13), _log(rng, 1, 64)
    p_hi = _log(rng, 1, 16384)
    p_lo = rng.randint(0, p_hi) if rng.random() < 0.7 else p_hi
    if op == "answer":
        slot = _log(rng, 1, 2000)
        room = 8 * 64 * 512 * 8 * 128 // (slot * kv * dim)
        samples = max(1, min(samples, room))
        groups = max(1, min(groups, room // samples, 2 * 32000 * 8 * 128 // (p_hi * kv * dim)))
        return dict(op=op, dtype=dtype, groups=groups, samples=samples, p_lo=p_lo, p_hi=p_hi,
                    lo=rng.randint(0, slot // 2), hi=slot, slot=slot, q_heads=heads, kv_heads=kv, dim=dim)
    hi = _log(rng, 1, 1500)
    lo = rng.randint(0, hi) if rng.random() < 0.7 else hi
    # Pairs of a row and a key that cost what the largest case does.
    room = 32 * 16 * 512 * 8448 // (hi * (p_hi + hi))
    heads = kv * max(1, min(heads, room) // kv)
    samples = max(1, min(samples, room // heads))
    groups = max(1, min(groups, room // heads // samples))
    return dict(op=op, dtype=dtype, groups=groups, samples=samples, p_lo=p_lo, p_hi=p_hi, lo=lo, hi=hi,
                q_heads=heads, kv_heads=kv, dim=dim)


def _lengths(n, lo, hi, salt):
    """The case's own lengths, the same for every seed; the longest is `hi`."""
    r = random.Random(977 * salt + 31 * n + lo + hi)
    got = [r.randint(lo, hi) for _ in range(n)]
    got[r.randrange(n)] = hi
    return got


def _offsets(lengths):
    at = [0]
    for x in lengths:
        at.append(at[-1] + x)
    return at


def _sizes(case):
    """(prefix lengths of the groups, own lengths of the sequences)."""
    n = case["groups"] * case["samples"]
    return (_lengths(case["groups"], case["p_lo"], case["p_hi"], 1),
            _lengths(n, case["lo"], case["hi"], 2))


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _randn(gen, shape, dtype):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    return out.normal_(generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": dict(case)}
    if case["op"] == "rotate":
        return _prepare_rotate(s, gen)
    if case["op"] == "beams":
        return _prepare_beams(s, gen)
    hq, hk, d, dtype = case["q_heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    p_len, own_len = _sizes(case)
    batch = len(own_len)
    s["groups"] = _i32([i * case["samples"] for i in range(case["groups"] + 1)])
    s["p_offsets"] = _i32(_offsets(p_len))
    s["p_k"], s["p_v"] = (_randn(gen, (sum(p_len), hk, d), dtype) for _ in range(2))
    s["p_most"] = max(p_len)
    if case["op"] == "answer":
        # Slots of one size; what lies behind a cache's last token is whatever
        # the memory held.
        slot = case["slot"]
        s["q_offsets"] = _i32(list(range(batch + 1)))
        s["k_offsets"] = _i32([i * slot for i in range(batch + 1)])
        s["k_lengths"] = _i32(own_len)
        s["q"] = _randn(gen, (batch, hq, d), dtype)
        s["k"], s["v"] = (_randn(gen, (batch * slot, hk, d), dtype) for _ in range(2))
        free = (torch.arange(slot, device="cuda")[None] >= s["k_lengths"][:, None]).reshape(-1)
        s["k"][free], s["v"][free] = float("nan"), float("inf")
        s["q_most"], s["k_most"] = 1, max(own_len)
    else:
        x = _randn(gen, (sum(own_len), hq + 2 * hk, d), dtype)  # slices of one projection
        s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        s["q_offsets"] = s["k_offsets"] = _i32(_offsets(own_len))
        s["d_out"] = _randn(gen, (sum(own_len), hq, d), dtype)
        s["q_most"] = s["k_most"] = max(own_len)
    return s


def _prepare_rotate(s, gen):
    case = s["case"]
    hq, hk, d, n, dtype = (case[x] for x in ("q_heads", "kv_heads", "dim", "rows", "dtype"))
    dtype = DTYPES[dtype]
    x = _randn(gen, (n, hq + 2 * hk, d), dtype)
    s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    for name in ("q_weight", "k_weight"):
        s[name] = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")
    half = case["turned"] // 2
    s["frequencies"] = (500000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()
    if case["cached"]:
        # Every sequence somewhere in its cache, near or far from its beginning.
        s["positions"] = torch.randint(0, 1 << 20, (n,), generator=gen, device="cuda")
        s["places"] = torch.arange(n, device="cuda") * case["slot"] + s["positions"] % case["slot"]
        s["k_cache"], s["v_cache"] = (_randn(gen, (n * case["slot"], hk, d), dtype) for _ in range(2))
    else:
        # Packed sequences; the second half of them deep inside long ones.
        at = torch.arange(n, device="cuda") % 8192
        far = torch.randint(0, 1 << 20, (1,), generator=gen, device="cuda")
        s["positions"] = torch.where(torch.arange(n, device="cuda") * 2 >= n, at + far, at)
        s["d_q_out"], s["d_k_out"] = (_randn(gen, (n, h, d), dtype) for h in (hq, hk))
    return s


def _prepare_beams(s, gen):
    """Logits as a trained model gives them: a few tokens of a row have most of
    its weight.  Beams' scores are such that no two of a group's best
    candidates of different beams are within 2e-5 of each other, which 32 bits
    would not tell apart."""
    case = s["case"]
    groups, beams, width, vocab = case["groups"], case["beams"], case["width"], case["vocab"]
    n, end = groups * beams, case["end"]
    x = torch.randn((n, vocab), generator=gen, device="cuda")
    few = min(vocab, 4)
    t = torch.randint(0, vocab, (n, few), generator=gen, device="cuda")
    x.scatter_add_(1, t, math.log(vocab) * torch.rand((n, few), generator=gen, device="cuda") + 1)
    s["logits"] = x.to(DTYPES[case["dtype"]])
    s["last"] = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    if end >= 0:
        finished = torch.rand(n, generator=gen, device="cuda") < 0.2
        s["last"] = torch.where(finished, end, torch.where(s["last"] == end, (end + 1) % vocab, s["last"]))
    z = torch.log_softmax(s["logits"].double() / case["temperature"], 1)
    if end >= 0:
        done = s["last"] == end
        z[done] = -math.inf
        z[done, end] = 0.0
    most = min(vocab, width + 1)
    z = z.topk(most, 1).values.view(groups, beams, most)
    scores = torch.zeros((groups, beams), device="cuda")
    close = torch.ones(groups, dtype=torch.bool, device="cuda")
    for _ in range(50):
        new = -4 - 3 * torch.rand((groups, beams), generator=gen, device="cuda")
        scores = torch.where(close[:, None], new, scores)
        best, at = (scores.double()[..., None] + z).view(groups, -1).sort(dim=1, descending=True)
        best, row = best[:, :width + 2], (at // most)[:, :width + 2]
        gap = best[:, :-1] - best[:, 1:]
        close = ((gap < 2e-5) & (row[:, 1:] != row[:, :-1])).any(1)
        if not bool(close.any()):
            break
    s["scores"] = scores.view(-1)
    slots = groups * width
    lengths = _i32(_lengths(slots, case["rows"] // 2, case["rows"], 3))
    s["states"] = _randn(gen, (case["outer"], slots, case["rows"], case["row"]), torch.bfloat16)
    s["lengths"] = lengths
    return s


# The plain forms.


def _turn(x, cos, sin, case):
    """Pairs of the first `turned` elements by the angles with these cosines and sines."""
    half = case["turned"] // 2
    cos, sin = cos[:, None], sin[:, None]
    if case["interleaved"]:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., 2 * half:]], -1)


def _plain_rotate(s):
    case = s["case"]
    angle = s["positions"].double()[:, None] * s["frequencies"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    got = {}
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "_weight"]
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        got[name + "_out"] = _turn(n * w, cos, sin, case).to(s[name].dtype)
        if case["cached"]:
            continue
        g = _turn(s[f"d_{name}_out"].float(), cos, -sin, case)
        got[f"d_{name}_weight"] = (g * n).sum((0, 1), dtype=torch.float64).float()
        u = g * w
        got["d_" + name] = (r * (u - n * (u * n).mean(-1, keepdim=True))).to(s[name].dtype)
    if case["cached"]:
        s["k_cache"][s["places"]], s["v_cache"][s["places"]] = got.pop("k_out"), s["v"]
        got["k_cache"], got["v_cache"] = s["k_cache"], s["v_cache"]
    return got


def _plain_attention(s):
    case = s["case"]
    hq, hk, dim, groups, samples = (case[x] for x in ("q_heads", "kv_heads", "dim", "groups", "samples"))
    share, batch, nq, nk, np_ = hq // hk, groups * samples, s["q_most"], s["k_most"], s["p_most"]
    q_len = s["q_offsets"][1:] - s["q_offsets"][:-1]
    k_len = s.get("k_lengths", s["k_offsets"][1:] - s["k_offsets"][:-1])
    p_len = s["p_offsets"][1:] - s["p_offsets"][:-1]
    on_q, on_k, on_p = (torch.arange(n, device="cuda") < x[:, None] for n, x in
                        ((nq, q_len), (nk, k_len), (np_, p_len)))

    def pad(x, offsets, on):  # [n, heads, rows, dim], zero behind the last row
        if not x.shape[0]:
            return torch.zeros((on.shape[0], x.shape[1], on.shape[1], dim), device="cuda")
        at = offsets[:-1, None] + torch.arange(on.shape[1], device="cuda")
        return torch.where(on[..., None, None], x[at.clamp(max=x.shape[0] - 1).long()].float(), 0.0).transpose(1, 2)

    def of_prefix(x):  # [batch, hk, share * nq, y] -> [groups, hk, samples * share * nq, y]
        return x.view(groups, samples, hk, share * nq, -1).transpose(1, 2).reshape(groups, hk, -1, x.shape[-1])

    def of_own(x):
        return x.view(groups, hk, samples, share * nq, -1).transpose(1, 2).reshape(batch, hk, share * nq, x.shape[-1])

    def rows(x, heads, on):
        return x.reshape(on.shape[0], heads, -1, dim).transpose(1, 2)[on]

    scale = dim ** -0.5
    q = pad(s["q"], s["q_offsets"], on_q).reshape(batch, hk, share * nq, dim)
    k, v = pad(s["k"], s["k_offsets"], on_k), pad(s["v"], s["k_offsets"], on_k)
    p_k, p_v = pad(s["p_k"], s["p_offsets"], on_p), pad(s["p_v"], s["p_offsets"], on_p)
    seen = on_q[:, :, None] & on_k[:, None, :]
    seen &= torch.arange(nk, device="cuda") <= (torch.arange(nq, device="cuda")[:, None]
                                                + (k_len - q_len)[:, None, None])
    a = torch.matmul(q, k.transpose(2, 3)) * scale
    a = a.view(batch, hk, share, nq, nk).masked_fill_(~seen[:, None, None], -math.inf).view(batch, hk, -1, nk)
    p = torch.matmul(of_prefix(q), p_k.transpose(2, 3)) * scale
    p.masked_fill_(~on_p[:, None, None], -math.inf)
    none = a.new_full((*a.shape[:3], 1), -math.inf)
    most = torch.maximum(a.amax(-1, keepdim=True) if nk else none,
                         of_own(p.amax(-1, keepdim=True)) if np_ else none)
    least = torch.where(most > -math.inf, most, 0.0)
    a, p = torch.exp(a - least), torch.exp(p - of_prefix(least))
    total = a.sum(-1, keepdim=True) + of_own(p.sum(-1, keepdim=True))
    by = torch.where(total > 0, 1 / total, 0.0)
    a, p = a * by, p * of_prefix(by)
    o = torch.matmul(a, v) + of_own(torch.matmul(p, p_v))
    lse = (most + torch.log(total)).view(batch, hq, nq).transpose(1, 2)[on_q].t().contiguous()
    got = {"out": rows(o, hq, on_q).to(s["q"].dtype), "lse": lse}
    if case["op"] == "answer":
        return got
    do = pad(s["d_out"], s["q_offsets"], on_q).reshape(batch, hk, share * nq, dim)
    p_do, p_q = of_prefix(do), of_prefix(q)
    got["d_v"] = rows(torch.matmul(a.transpose(2, 3), do), hk, on_k).to(s["q"].dtype)
    got["d_p_v"] = rows(torch.matmul(p.transpose(2, 3), p_do), hk, on_p).to(s["q"].dtype)
    delta = (do * o).sum(-1, keepdim=True)
    a = a * (torch.matmul(do, v.transpose(2, 3)) - delta) * scale
    p = p * (torch.matmul(p_do, p_v.transpose(2, 3)) - of_prefix(delta)) * scale
    d_q = torch.matmul(a, k) + of_own(torch.matmul(p, p_k))
    got["d_q"] = rows(d_q, hq, on_q).to(s["q"].dtype)
    got["d_k"] = rows(torch.matmul(a.transpose(2, 3), q), hk, on_k).to(s["q"].dtype)
    got["d_p_k"] = rows(torch.matmul(p.transpose(2, 3), p_q), hk, on_p).to(s["q"].dtype)
    return got


def _plain_beams(s):
    case = s["case"]
    groups, beams, width, vocab = case["groups"], case["beams"], case["width"], case["vocab"]
    x = s["logits"].float() / case["temperature"]
    x = x - x.amax(1, keepdim=True)
    base = s["scores"].double() - torch.log(torch.exp(x).sum(1, dtype=torch.float64))
    del x
    z = s["logits"].double() / case["temperature"]
    z = z - z.amax(1, keepdim=True) + base[:, None]
    if case["end"] >= 0:  # a finished beam stays as it is
        done = s["last"] == case["end"]
        z.masked_fill_(done[:, None], -math.inf)
        z[:, case["end"]] = torch.where(done, s["scores"].double(), z[:, case["end"]])
    z = z.view(groups, beams * vocab)
    score, at = z.sort(dim=1, descending=True, stable=True)
    score, at = score[:, :width], at[:, :width]
    del z
    short = width - score.shape[1]
    if short > 0:
        score = torch.cat([score, score.new_full((groups, short), -math.inf)], 1)
        at = torch.cat([at, at.new_zeros((groups, short))], 1)
    on = score > -math.inf
    beam, token = torch.where(on, at // vocab, -1), torch.where(on, at % vocab, -1)
    if case["stay"]:
        # A beam's first continuation takes its slot, the others the slots that are left.
        rank = torch.arange(width, device="cuda")
        first = on & ~((beam[:, :, None] == beam[:, None, :]) & (rank[None, :] < rank[:, None])).any(2)
        used = torch.zeros((groups, beams + 1), dtype=torch.bool, device="cuda")
        used.scatter_(1, torch.where(first, beam, beams), True)
        left = used[:, :beams].long().sort(dim=1, stable=True).indices  # free slots first
        nth = (~first).long().cumsum(1) - 1
        slot = torch.where(first, beam, left.gather(1, nth.clamp(min=0)))
        order = slot.argsort(1)
        beam, token, score = beam.gather(1, order), token.gather(1, order), score.gather(1, order)
    parents = torch.where(beam >= 0, beam + torch.arange(groups, device="cuda")[:, None] * beams, -1)
    parents = parents.int().view(-1)
    if beams == width:
        p = parents.clamp(min=0).long()
        move = (torch.arange(case["rows"], device="cuda") < s["lengths"][p][:, None]) & (parents >= 0)[:, None]
        for x in s["states"]:
            x.copy_(torch.where(move[..., None], x[p], x))
    return {"scores": score.float().view(-1), "parents": parents, "tokens": token.view(-1), "states": s["states"]}


# The package's operators.


def _own(s):
    import paper_2607_22242_amd as S

    case, op = s["case"], s["case"]["op"]
    if op == "rotate":
        how = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, interleaved=case["interleaved"])
        if case["cached"]:
            q_out, _, _ = S.sched_norm_rotate(s["q"], s["k"], s["positions"], s["frequencies"], v=s["v"],
                                              places=s["places"], k_out=s["k_cache"], v_out=s["v_cache"], **how)
            return {"q_out": q_out, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        q_out, k_out = S.sched_norm_rotate(s["q"], s["k"], s["positions"], s["frequencies"], **how)
        d_q, d_k, d_qw, d_kw = S.sched_norm_rotate_grad(s["q"], s["k"], s["d_q_out"], s["d_k_out"],
                                                        s["positions"], s["frequencies"], **how)
        return {"q_out": q_out, "d_q_weight": d_qw, "d_q": d_q, "k_out": k_out, "d_k_weight": d_kw, "d_k": d_k}
    if op == "beams":
        scores, parents, tokens = S.sched_beam_select(
            s["logits"], s["scores"], case["beams"], case["width"], last=s["last"], end_token=case["end"],
            temperature=case["temperature"], stay=case["stay"])
        if case["beams"] == case["width"]:
            S.sched_beam_reorder(s["states"], parents, case["beams"], lengths=s["lengths"])
        return {"scores": scores, "parents": parents, "tokens": tokens, "states": s["states"]}
    args = (s["q"], s["k"], s["v"], s["p_k"], s["p_v"])
    where = (s["q_offsets"], s["k_offsets"], s["p_offsets"], s["groups"])
    if op == "answer":
        out, lse = S.sched_shared_attention(*args, *where, k_lengths=s["k_lengths"])
        return {"out": out, "lse": lse}
    out, lse = S.sched_shared_attention(*args, *where)
    d_q, d_k, d_v, d_p_k, d_p_v = S.sched_shared_attention_grad(*args, out, lse, s["d_out"], *where)
    return {"out": out, "lse": lse, "d_v": d_v, "d_p_v": d_p_v, "d_q": d_q, "d_k": d_k, "d_p_k": d_p_k}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "rotate":
        return _plain_rotate(state)
    return _plain_beams(state) if op == "beams" else _plain_attention(state)


def work(case):
    op, b = case["op"], BYTES[case["dtype"]]
    if op == "rotate":
        n, d, hq, hk = case["rows"], case["dim"], case["q_heads"], case["kv_heads"]
        x = n * (hq + hk) * d
        if case["cached"]:
            return {"bytes": (2 * x + 2 * n * hk * d) * b + 16 * n, "flops": 8 * x}
        # Forward in and out; backward in, the gradient in and out.
        return {"bytes": 5 * x * b + 16 * n, "flops": 24 * x}
    if op == "beams":
        n, slots = case["groups"] * case["beams"], case["groups"] * case["width"]
        # Finished beams' logits are not read.  Of these inputs' beams six in
        # ten (of those that stay), or nearly all, get another's state, which
        # is read once for all that get it.
        read = n * case["vocab"] * b * (0.8 if case["end"] >= 0 else 1.0)
        moved = 0.0
        if case["beams"] == case["width"] and case["beams"] > 1:
            moved = (0.6 + 0.35) if case["stay"] else (0.95 + 0.4)
        states = case["outer"] * sum(_lengths(slots, case["rows"] // 2, case["rows"], 3)) * case["row"] * 2
        return {"bytes": int(read + moved * states) + 16 * (n + slots), "flops": 6 * n * case["vocab"]}
    p_len, own_len = _sizes(case)
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    pairs, nq = 0, 0
    for i, m in enumerate(own_len):
        p = p_len[i // case["samples"]]
        pairs += p + m if op == "answer" else m * p + m * (m + 1) // 2
        nq += 1 if op == "answer" else m
    read = (nq * hq + 2 * (sum(own_len) + sum(p_len)) * hk) * dim * b
    if op == "answer":
        return {"bytes": read + nq * hq * (dim * b + 4), "flops": 4 * pairs * hq * dim}
    # Forward two products, backward five (the scores are computed again).
    return {"bytes": 2 * read + nq * hq * (2 * dim * b + 4), "flops": 14 * pairs * hq * dim}


# The definitions in 64 bits.


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return _exact_rotate(s)
    return _exact_beams(s) if case["op"] == "beams" else _exact_attention(s)


def _exact_rotate(s):
    case = s["case"]
    half, got = case["turned"] // 2, {}
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * s["frequencies"].double())[:, None]
    for name in ("q", "k"):
        x, w = s[name].double().requires_grad_(), s[name + "_weight"].double().requires_grad_()
        y = x / torch.sqrt(torch.mean(x ** 2, -1, keepdim=True) + EPS) * w
        head = y[..., :2 * half]
        if case["interleaved"]:
            z = torch.view_as_complex(head.reshape(*head.shape[:-1], half, 2).contiguous()) * turn
            head = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(head[..., :half], head[..., half:]) * turn
            head = torch.cat([z.real, z.imag], -1)
        y = torch.cat([head, y[..., 2 * half:]], -1)
        got[name + "_out"] = y.detach()
        if not case["cached"]:
            d, dw = torch.autograd.grad(y, (x, w), s[f"d_{name}_out"].double())
            got[f"d_{name}_weight"], got["d_" + name] = dw, d
    if case["cached"]:
        k_out, places = got.pop("k_out"), s["places"].tolist()
        for name, rows in (("k_cache", k_out), ("v_cache", s["v"].double())):
            cache = s[name].double()
            for i, at in enumerate(places):
                cache[at] = rows[i]
            got[name] = cache
    return got


def _exact_attention(s):
    case = s["case"]
    q_at, k_at, p_at = (s[x].tolist() for x in ("q_offsets", "k_offsets", "p_offsets"))
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    share, answer = hq // hk, case["op"] == "answer"
    lengths = s["k_lengths"].tolist() if answer else [b - a for a, b in zip(k_at, k_at[1:])]
    zeros = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    got = {"out": zeros(s["q"]),
           "lse": torch.full((hq, s["q"].shape[0]), -math.inf, dtype=torch.float64, device="cuda")}
    if not answer:
        got.update(d_v=zeros(s["v"]), d_p_v=zeros(s["p_v"]), d_q=zeros(s["q"]), d_k=zeros(s["k"]),
                   d_p_k=zeros(s["p_k"]))
    for b, own_n in enumerate(lengths):
        g = b // case["samples"]
        rq, rk, rp = slice(q_at[b], q_at[b + 1]), slice(k_at[b], k_at[b] + own_n), slice(p_at[g], p_at[g + 1])
        nq, before = rq.stop - rq.start, rp.stop - rp.start
        if not nq or not own_n + before:
            continue
        # All keys of the sequence, those of its prefix first: [hk, keys, dim].
        k = torch.cat([s["p_k"][rp], s["k"][rk]]).double().transpose(0, 1).contiguous()
        v = torch.cat([s["p_v"][rp], s["v"][rk]]).double().transpose(0, 1).contiguous()
        q = s["q"][rq].double().view(nq, hk, share, dim).permute(1, 2, 0, 3).reshape(hk, -1, dim)
        a = (q @ k.transpose(1, 2)).view(hk, share, nq, -1) / math.sqrt(dim)
        i, j = torch.arange(nq, device="cuda")[:, None], torch.arange(own_n, device="cuda")
        a[..., before:].masked_fill_(j > i + (own_n - nq), -math.inf)
        lse = torch.logsumexp(a, -1, keepdim=True)
        p = torch.where(lse > -math.inf, torch.exp(a - lse), 0.0).view(hk, share * nq, -1)
        o = p @ v

        def out_of(x):
            return x.view(hk, share, nq, dim).permute(2, 0, 1, 3).reshape(nq, hq, dim)

        got["out"][rq] = out_of(o)
        got["lse"][:, rq] = lse.view(hq, nq)
        if answer:
            continue
        do = s["d_out"][rq].double().view(nq, hk, share, dim).permute(1, 2, 0, 3).reshape(hk, -1, dim)
        dv = (p.transpose(1, 2) @ do).transpose(0, 1)
        ds = p * (do @ v.transpose(1, 2) - (do * o).sum(-1, keepdim=True)) / math.sqrt(dim)
        dk = (ds.transpose(1, 2) @ q).transpose(0, 1)
        got["d_q"][rq] = out_of(ds @ k)
        got["d_k"][rk], got["d_v"][rk] = dk[before:], dv[before:]
        got["d_p_k"][rp] += dk[:before]
        got["d_p_v"][rp] += dv[:before]
    return got


def _exact_beams(s):
    case = s["case"]
    groups, beams, width, vocab, end = (case[x] for x in ("groups", "beams", "width", "vocab", "end"))
    scores, parents, tokens = [], [], []
    last = s["last"].tolist()
    for g in range(groups):
        rows = range(g * beams, (g + 1) * beams)
        found = []  # (score, beam, token), each beam's best
        for i in rows:
            start = float(s["scores"][i])
            if end >= 0 and last[i] == end:
                found.append((-start, i, end))
                continue
            z = torch.log_softmax(s["logits"][i].double() / case["temperature"], 0) + start
            # All that reach the beam's `width`-th best, ties among them.
            best = z.topk(min(width, vocab)).values[-1]
            at = (z >= best).nonzero()[:, 0]
            found += [(-x, i, t) for x, t in zip(z[at].tolist(), at.tolist())]
        found = sorted(found)[:width]
        slots = [None] * width
        if case["stay"]:
            rest = []
            for c in found:
                if slots[c[1] - rows.start] is None:
                    slots[c[1] - rows.start] = c
                else:
                    rest.append(c)
            for i in range(width):
                if slots[i] is None and rest:
                    slots[i] = rest.pop(0)
        else:
            slots[:len(found)] = found
        for c in slots:
            scores.append(-math.inf if c is None else -c[0])
            parents.append(-1 if c is None else c[1])
            tokens.append(-1 if c is None else c[2])
    states = s["states"].clone()
    if beams == width:
        lengths = s["lengths"].tolist()
        for i, p in enumerate(parents):
            if p >= 0:
                states[:, i, :lengths[p]] = s["states"][:, p, :lengths[p]]
    return {"scores": torch.tensor(scores, dtype=torch.float64, device="cuda"), "parents": _i32(parents),
            "tokens": torch.tensor(tokens, dtype=torch.int64, device="cuda"), "states": states}
