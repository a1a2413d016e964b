"""The operators of a mapping agent whose speed matters, one dict of plain values each.

The search scores device mappings; a language model proposes them (Section 3.3)
and is trained on what the scores say.  A case is one pass through the
operators of one step of that training, or of the agent's answering, the way a
program calls them: tensors on the GPU, ragged sequences packed one after the
other, int32 offsets on the device.

policy      group advantages from makespans, then the clipped policy loss with
            a KL term from the logits, with the logits' gradient
preference  log-probabilities of the answers' tokens, the loss over pairs of a
            better and a worse mapping, and the logits' gradient
embed       the lookup with scaling, and its gradient by sorted tokens
attend      attention over packed sequences and its backward pass
decode      attention of single tokens over a cache

`run` computes these in elementary torch operations in 32 bits, or by the
package's operators where `own` is true; `exact` in 64 bits, from the
definitions.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
NEVER = (1 << 63) - 1  # the makespan of an infeasible mapping


def listed():
    return [
        # One round's policy update of an agent that answers with a mode per
        # tool: 13 scenarios x 64 sampled mappings of 14 tools (the batched
        # workload), three classes, a call's latency.
        dict(name="policy modes", op="policy", dtype="f32", vocab=3, groups=13, samples=64,
             lo=14, hi=14, temperature=1.0, mean="tokens"),
        # An ordinary update of a small language model: 8 scenarios x 8 answers
        # of 20 to 120 tokens, an odd vocabulary.
        dict(name="policy 32003", op="policy", dtype="bf16", vocab=32003, groups=8, samples=8,
             lo=20, hi=120, temperature=0.7, mean="sequences"),
        # The largest update: a vocabulary of 131072 and about 8,000 answer
        # tokens, 2 GB of logits.
        dict(name="policy 131072", op="policy", dtype="bf16", vocab=131072, groups=8, samples=16,
             lo=30, hi=96, temperature=1.0, mean="tokens"),
        # Pairs of a better and a worse mapping of 19 tools, spelled in tokens
        # of a small vocabulary.
        dict(name="pairs 257", op="preference", dtype="f16", vocab=257, pairs=40, lo=12, hi=64,
             temperature=1.0, smoothing=0.0),
        # An ordinary preference step: 48 pairs of reasoned answers.
        dict(name="pairs 50021", op="preference", dtype="bf16", vocab=50021, pairs=48, lo=40,
             hi=300, temperature=1.0, smoothing=0.1),
        # Tool cards of one workflow as bucketed tokens, in 32 bits.
        dict(name="embed cards", op="embed", dtype="f32", vocab=512, dim=64, tokens=1001,
             zipf=0.6, accumulate=False),
        # A micro-batch that adds to the 32-bit gradient of earlier ones.
        dict(name="embed accumulate", op="embed", dtype="bf16", vocab=50021, dim=2056,
             tokens=8191, zipf=1.0, accumulate=True),
        # The largest: 65,536 tokens of a large vocabulary, dense gradient.
        dict(name="embed 131072", op="embed", dtype="bf16", vocab=131072, dim=4096,
             tokens=65536, zipf=1.0, accumulate=False),
        # The agent answering: one new token for each of 48 workflows, caches
        # of 1 to 16,384 tokens in slots of one size.
        dict(name="decode 48", op="decode", dtype="bf16", batch=48, q_heads=32, kv_heads=8,
             dim=128, slot=16384, lo=1, hi=16384),
        # Prompts of tool cards and answers, 64 short ragged sequences.
        dict(name="attend short", op="attend", dtype="f16", batch=64, q_heads=8, kv_heads=8,
             dim=64, lo=40, hi=260, causal=True, cross=0.0),
        # An ordinary training step: ragged sequences, shared key heads.
        dict(name="attend ragged", op="attend", dtype="bf16", batch=8, q_heads=16, kv_heads=4,
             dim=128, lo=300, hi=2500, causal=True, cross=0.0),
        # The largest: one long sequence.
        dict(name="attend 8192", op="attend", dtype="bf16", batch=1, q_heads=32, kv_heads=8,
             dim=128, lo=8192, hi=8192, causal=True, cross=0.0),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["policy", "policy", "preference", "embed", "embed", "decode", "attend",
                     "attend", "attend"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    if op == "policy":
        vocab, lo = _log(rng, 2, 131072), rng.randint(1, 60)
        hi = lo + rng.randint(0, 90)
        room = 8064 * 131072 * 2 // (vocab * BYTES[dtype])  # rows that cost what the largest does
        groups = _log(rng, 1, 13)
        samples = max(2, min(_log(rng, 2, 64), room // (groups * hi)))
        groups = max(1, min(groups, room // (samples * hi)))
        return dict(op=op, dtype=dtype, vocab=vocab, groups=groups, samples=samples, lo=lo, hi=hi,
                    temperature=rng.choice([0.7, 1.0, 1.3]),
                    mean=rng.choice(["tokens", "sequences"]))
    if op == "preference":
        vocab, lo = _log(rng, 3, 131072), rng.randint(1, 100)
        hi = lo + rng.randint(0, 200)
        room = 8000 * 131072 * 2 // (vocab * BYTES[dtype] * 2)
        pairs = max(1, min(_log(rng, 1, 100), room // (2 * hi)))
        return dict(op=op, dtype=dtype, vocab=vocab, pairs=pairs, lo=lo, hi=hi,
                    temperature=rng.choice([0.7, 1.0, 1.3]), smoothing=rng.choice([0.0, 0.1]))
    if op == "embed":
        dim = _log(rng, 8, 4096)
        dim = dim if rng.random() < 0.3 else max(8, dim // 8 * 8)
        return dict(op=op, dtype=dtype, vocab=_log(rng, 3, 100000), dim=dim,
                    tokens=_log(rng, 1, 60000), zipf=rng.choice([0.0, 0.6, 1.0, 1.3]),
                    accumulate=rng.random() < 0.4)
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 8])
    dim = rng.choice([16, 40, 64, 64, 80, 96, 120, 128, 128, 128])
    dtype = rng.choice(["f16", "bf16", "bf16"])
    if op == "decode":
        slot = _log(rng, 1, 20000)
        batch = max(1, min(_log(rng, 1, 64), 48 * 16384 * 8 * 128 // (slot * kv * dim)))
        return dict(op=op, dtype=dtype, batch=batch, q_heads=heads, kv_heads=kv, dim=dim,
                    slot=slot, lo=rng.randint(0, slot // 2), hi=slot)
    hi = _log(rng, 1, 8192)
    lo = rng.randint(0, hi) if rng.random() < 0.7 else hi
    causal = rng.random() < 0.75
    # Pairs of tokens that cost what the largest does; half are seen where it is causal.
    room = 32 * 8192 ** 2 // (2 - causal) // (hi * hi)
    heads = kv * max(1, min(heads, room) // kv)
    return dict(op=op, dtype=dtype, batch=max(1, min(_log(rng, 1, 64), room // heads)),
                q_heads=heads, kv_heads=kv, dim=dim, lo=lo, hi=hi, causal=causal,
                cross=rng.choice([0.0, 0.0, 0.5]))


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
    """Lengths of the packed sequences of a case: (queries, keys) or (answers, None)."""
    op = case["op"]
    if op == "policy":
        return _lengths(case["groups"] * case["samples"], case["lo"], case["hi"], 1), None
    if op == "preference":
        return _lengths(2 * case["pairs"], case["lo"], case["hi"], 2), None
    if op == "decode":
        return [1] * case["batch"], _lengths(case["batch"], case["lo"], case["hi"], 3)
    q = _lengths(case["batch"], case["lo"], case["hi"], 4)
    if not case["cross"]:
        return q, q
    return q, [max(0, int(x * case["cross"])) if i % 2 else x for i, x in enumerate(q)]


def _ignored(length):
    """Tokens at the head of an answer that carry no loss (its prompt's last ones)."""
    return length // 16


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _noise(gen, shape, lo, hi):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def _answers(case, gen, lengths):
    """Logits as a trained model gives them (most of a row's weight on the
    answer), the answers' tokens with -1 where there is no loss, and the
    log-probabilities of the tokens."""
    n, vocab, dtype = sum(lengths), case["vocab"], DTYPES[case["dtype"]]
    tokens = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    logits = torch.empty((n, vocab), dtype=dtype, device="cuda")
    logp = torch.empty(n, dtype=torch.float32, device="cuda")
    step = max(1, (1 << 27) // vocab)
    for a in range(0, n, step):
        x = torch.randn((min(step, n - a), vocab), generator=gen, device="cuda") * 2
        t = tokens[a:a + step, None]
        x.scatter_add_(1, t, torch.full_like(x[:, :1], math.log(vocab)))
        logits[a:a + step] = x.to(dtype)
        x = logits[a:a + step].float() / case["temperature"]
        logp[a:a + step] = (x.gather(1, t) - torch.logsumexp(x, 1, keepdim=True))[:, 0]
    offsets = _offsets(lengths)
    skip = [i for a, x in zip(offsets, lengths) for i in range(a, a + _ignored(x))]
    if skip:
        tokens[torch.tensor(skip, device="cuda")] = -1
    return logits, tokens, logp, _i32(offsets)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    s = {"case": dict(case)}
    if op in ("policy", "preference"):
        lengths, _ = _sizes(case)
        s["logits"], s["tokens"], logp, s["offsets"] = _answers(case, gen, lengths)
        n = len(logp)
    if op == "policy":
        # Off-policy by up to a third, past the clip range on both sides for
        # some tokens; no ratio lies on a clip bound, where the gradient jumps.
        shift = _noise(gen, n, -0.3, 0.3)
        ratio = torch.exp(shift)
        near = ((ratio - 0.8).abs() < 1e-3) | ((ratio - 1.25).abs() < 1e-3)
        s["old_logp"] = logp - torch.where(near, shift * 0.5, shift)
        s["ref_logp"] = logp + _noise(gen, n, -0.4, 0.4)
        count = case["groups"] * case["samples"]
        made = torch.randint(400_000, 2_000_000, (count,), generator=gen, device="cuda")
        made[torch.rand(count, generator=gen, device="cuda") < 0.1] = NEVER
        s["makespans"] = made
        s["groups"] = _i32([i * case["samples"] for i in range(case["groups"] + 1)])
        s["limits"] = torch.full((case["groups"],), 2_500_000, dtype=torch.int64, device="cuda")
    elif op == "preference":
        s["ref_logp"] = logp + _noise(gen, n, -0.4, 0.4)
    elif op == "embed":
        vocab, dim, n, dtype = case["vocab"], case["dim"], case["tokens"], DTYPES[case["dtype"]]
        s["table"] = torch.randn((vocab, dim), generator=gen, device="cuda").to(dtype)
        s["d_rows"] = torch.randn((n, dim), generator=gen, device="cuda").to(dtype)
        # Frequencies fall as rank ** -zipf; ranks are spread over the vocabulary.
        w = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** -case["zipf"]
        u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * w.sum()
        rank = torch.searchsorted(torch.cumsum(w, 0), u).clamp_(max=vocab - 1)
        tokens = torch.randperm(vocab, generator=gen, device="cuda")[rank]
        tokens[::29] = -1 if n > 29 else tokens[0]  # padding
        s["tokens"] = tokens
        s["scale"] = math.sqrt(dim)
        if case["accumulate"]:
            s["acc"] = torch.randn((vocab, dim), generator=gen, device="cuda")
    else:
        q_len, k_len = _sizes(case)
        hq, hk, d, dtype = case["q_heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]

        def rand(rows, heads):
            return torch.randn((rows, heads, d), generator=gen, device="cuda").to(dtype)

        s["q_offsets"] = _i32(_offsets(q_len))
        if op == "decode":
            # Slots of one size; what lies behind a cache's last token is
            # whatever the memory held.
            slot, batch = case["slot"], case["batch"]
            s["k_offsets"] = _i32([i * slot for i in range(batch + 1)])
            s["k_lengths"] = _i32(k_len)
            s["q"], s["k"], s["v"] = rand(batch, hq), rand(batch * slot, hk), rand(batch * slot, hk)
            free = (torch.arange(slot, device="cuda")[None] >= s["k_lengths"][:, None]).reshape(-1)
            s["k"][free], s["v"][free] = float("nan"), float("inf")
            s["q_most"], s["k_most"] = 1, slot
        else:
            s["k_offsets"] = _i32(_offsets(k_len))
            if q_len == k_len:  # slices of one projection
                x = rand(sum(q_len), hq + 2 * hk)
                s["q"], s["k"], s["v"] = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
            else:
                s["q"], s["k"], s["v"] = rand(sum(q_len), hq), rand(sum(k_len), hk), rand(sum(k_len), hk)
            s["d_out"] = rand(sum(q_len), hq)
            s["q_most"], s["k_most"] = max(q_len), max(k_len)
    return s


# The plain forms.


def _plain_logprobs(s):
    """(log-probabilities of the tokens, probabilities, rows with loss); 0 where there is none."""
    x = s["logits"].float() / s["case"]["temperature"]
    on = s["tokens"] >= 0
    t = s["tokens"].clamp(min=0)[:, None]
    x = x - x.amax(1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    logp = torch.where(on, (x.gather(1, t) - torch.log(total))[:, 0], 0.0)
    return logp, e / total, on


def _plain_d_logits(s, d_logp, p, on):
    g = torch.where(on, d_logp, 0.0)[:, None] / s["case"]["temperature"]
    d = -p * g
    d.scatter_add_(1, s["tokens"].clamp(min=0)[:, None], g)
    return d.to(s["logits"].dtype)


def _plain_policy(s):
    case = s["case"]
    m = torch.minimum(s["makespans"], s["limits"].repeat_interleave(case["samples"])).float()
    m = m.view(case["groups"], case["samples"])
    mean = m.mean(1, keepdim=True)
    std = ((m - mean) ** 2).mean(1, keepdim=True).sqrt()
    adv = torch.where(std > 0, (mean - m) / std, 0.0).view(-1)
    lengths = (s["offsets"][1:] - s["offsets"][:-1]).long()
    n = s["tokens"].numel()
    seq = torch.repeat_interleave(torch.arange(adv.numel(), device="cuda"), lengths, output_size=n)
    logp, p, on = _plain_logprobs(s)
    counts = torch.zeros(adv.numel(), device="cuda").index_add_(0, seq, on.float())
    if case["mean"] == "tokens":
        weight = (on.float() / counts.sum().clamp(min=1))
    else:
        weight = on.float() / (counts[seq].clamp(min=1) * (counts > 0).sum().clamp(min=1))
    a = adv[seq]
    ratio = torch.exp(logp - s["old_logp"])
    free, held = -a * ratio, -a * ratio.clamp(0.8, 1.25)
    gap = s["ref_logp"] - logp
    kl = torch.exp(gap) - gap - 1
    losses = torch.where(on, weight * (torch.maximum(free, held) + 0.04 * kl), 0.0)
    d = weight * (torch.where(free >= held, free, 0.0) + 0.04 * (1 - torch.exp(gap)))
    return {"loss": losses.sum().view(1), "losses": losses, "logp": logp,
            "d_logits": _plain_d_logits(s, d, p, on)}


def _plain_preference(s):
    case = s["case"]
    logp, p, on = _plain_logprobs(s)
    lengths = (s["offsets"][1:] - s["offsets"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(2 * case["pairs"], device="cuda"), lengths,
                                  output_size=logp.numel())
    gain = torch.where(on, logp - s["ref_logp"], 0.0)
    total = torch.zeros(2 * case["pairs"], device="cuda").index_add_(0, seq, gain)
    margin = 0.1 * (total[0::2] - total[1::2])
    soft = torch.log1p(torch.exp(-margin.abs()))
    up, down = soft - margin.clamp(max=0), soft + margin.clamp(min=0)  # -log sigmoid(+-margin)
    eps = case["smoothing"]
    loss = ((1 - eps) * up + eps * down).mean().view(1)
    d = (eps - 1) / (1 + torch.exp(margin)) + eps / (1 + torch.exp(-margin))
    d = 0.1 * d / case["pairs"]
    d_logp = torch.where(on, torch.stack([d, -d], 1).view(-1)[seq], 0.0)
    return {"loss": loss, "margins": margin, "logp": logp, "d_logp": d_logp,
            "d_logits": _plain_d_logits(s, d_logp, p, on)}


def _plain_embed(s):
    on = (s["tokens"] >= 0)[:, None]
    t = s["tokens"].clamp(min=0)
    rows = torch.where(on, s["table"][t].float() * s["scale"], 0.0).to(s["table"].dtype)
    g = torch.where(on, s["d_rows"].float(), 0.0)
    d = torch.zeros(s["table"].shape, device="cuda").index_add_(0, t, g) * s["scale"]
    if "acc" in s:
        s["acc"] += d
        return {"rows": rows, "d_table": s["acc"]}
    return {"rows": rows, "d_table": d.to(s["table"].dtype)}


def _plain_attention(s):
    case = s["case"]
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    nq, nk, batch = s["q_most"], s["k_most"], case["batch"]
    q_len = s["q_offsets"][1:] - s["q_offsets"][:-1]
    k_len = s.get("k_lengths", s["k_offsets"][1:] - s["k_offsets"][:-1])
    iq, ik = torch.arange(nq, device="cuda"), torch.arange(nk, device="cuda")
    on_q, on_k = iq < q_len[:, None], ik < k_len[:, None]

    def pad(x, offsets, i, on):  # [batch, heads, rows, dim], zero behind the last row
        if not x.shape[0]:
            return torch.zeros((batch, x.shape[1], len(i), dim), device="cuda")
        at = (offsets[:-1, None] + i).clamp(max=x.shape[0] - 1).long()
        return torch.where(on[..., None, None], x[at].float(), 0.0).transpose(1, 2)

    def group(x):  # the query heads that share a key head, one after the other
        return x.reshape(batch, hk, hq // hk * nq, dim)

    def rows(x, heads, on):
        return x.reshape(batch, heads, -1, dim).transpose(1, 2)[on]

    scale = dim ** -0.5
    q = group(pad(s["q"], s["q_offsets"], iq, on_q))
    k, v = pad(s["k"], s["k_offsets"], ik, on_k), pad(s["v"], s["k_offsets"], ik, on_k)
    seen = on_q[:, :, None] & on_k[:, None, :]
    if case.get("causal", True):
        seen &= ik <= iq[:, None] + (k_len - q_len)[:, None, None]
    a = torch.matmul(q, k.transpose(2, 3)).view(batch, hk, hq // hk, nq, nk) * scale
    a.masked_fill_(~seen[:, None, None], -math.inf)
    most = a.amax(-1, keepdim=True) if nk else a.new_full((*a.shape[:-1], 1), -math.inf)
    a = torch.exp(a - torch.where(most > -math.inf, most, 0.0))
    total = a.sum(-1, keepdim=True)
    lse = (most + torch.log(total)).view(batch, hq, nq).transpose(1, 2)[on_q].t().contiguous()
    p = (a / torch.where(total > 0, total, 1.0)).view(batch, hk, -1, nk)
    del a
    o = torch.matmul(p, v)
    got = {"out": rows(o, hq, on_q).to(s["q"].dtype), "lse": lse}
    if case["op"] == "decode":
        return got
    do = group(pad(s["d_out"], s["q_offsets"], iq, on_q))
    got["d_v"] = rows(torch.matmul(p.transpose(2, 3), do), hk, on_k).to(s["v"].dtype)
    ds = p * (torch.matmul(do, v.transpose(2, 3)) - (do * o).sum(-1, keepdim=True)) * scale
    got["d_q"] = rows(torch.matmul(ds, k), hq, on_q).to(s["q"].dtype)
    got["d_k"] = rows(torch.matmul(ds.transpose(2, 3), q), hk, on_k).to(s["k"].dtype)
    return got


# The package's operators.


def _own(s):
    import paper_2607_22242_amd as S

    case, op = s["case"], s["case"]["op"]
    if op == "policy":
        adv, weights = S.sched_group_advantages(s["makespans"], s["limits"], s["groups"],
                                                s["offsets"], s["tokens"], mean=case["mean"])
        loss, losses, logp, d_logits = S.sched_policy_loss(
            s["logits"], s["tokens"], s["old_logp"], s["ref_logp"], adv, weights, clip_low=0.2,
            clip_high=0.25, kl_weight=0.04, temperature=case["temperature"])
        return {"loss": loss, "losses": losses, "logp": logp, "d_logits": d_logits}
    if op == "preference":
        logp = S.sched_token_logprobs(s["logits"], s["tokens"], temperature=case["temperature"])
        loss, margins, d_logp = S.sched_preference_loss(logp, s["ref_logp"], s["tokens"],
                                                        s["offsets"], beta=0.1,
                                                        smoothing=case["smoothing"])
        d_logits = S.sched_token_logprobs_grad(s["logits"], s["tokens"], logp, d_logp,
                                               temperature=case["temperature"])
        return {"loss": loss, "margins": margins, "logp": logp, "d_logp": d_logp,
                "d_logits": d_logits}
    if op == "embed":
        rows = S.sched_embed(s["table"], s["tokens"], scale=s["scale"])
        if "acc" in s:
            d = S.sched_embed_grad(s["d_rows"], s["tokens"], case["vocab"], scale=s["scale"],
                                   out=s["acc"], accumulate=True)
        else:
            d = S.sched_embed_grad(s["d_rows"], s["tokens"], case["vocab"], scale=s["scale"])
        return {"rows": rows, "d_table": d}
    out, lse = S.sched_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"],
                                 k_lengths=s.get("k_lengths"), causal=case.get("causal", True))
    if op == "decode":
        return {"out": out, "lse": lse}
    d_q, d_k, d_v = S.sched_attention_grad(s["q"], s["k"], s["v"], out, lse, s["d_out"],
                                           s["q_offsets"], s["k_offsets"],
                                           causal=case.get("causal", True))
    return {"out": out, "lse": lse, "d_q": d_q, "d_k": d_k, "d_v": d_v}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "policy":
        return _plain_policy(state)
    if op == "preference":
        return _plain_preference(state)
    if op == "embed":
        return _plain_embed(state)
    return _plain_attention(state)


def work(case):
    op, b = case["op"], BYTES[case["dtype"]]
    q_len, k_len = _sizes(case) if op != "embed" else (None, None)
    if op in ("policy", "preference"):
        n, vocab = sum(q_len), case["vocab"]
        on = n - sum(map(_ignored, q_len))
        # Logits read where a token has a loss, their gradient written
        # everywhere; per token its id and a few 32-bit values.
        per = 8 + (2 + 2) * 4 if op == "policy" else 8 + (1 + 2) * 4
        return {"bytes": (on + n) * vocab * b + n * per + len(q_len) * 12, "flops": 8 * on * vocab}
    if op == "embed":
        n, dim, vocab = case["tokens"], case["dim"], case["vocab"]
        # At most as many table rows are read, or touched in place, as there are tokens or rows.
        rows = min(n, vocab)
        table = 2 * rows * dim * 4 if case["accumulate"] else vocab * dim * b
        return {"bytes": rows * dim * b + 2 * n * dim * b + table + 2 * n * 8,
                "flops": 2 * n * dim}
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    nq, nk = sum(q_len), sum(k_len)
    pairs = 0
    for q, k in zip(q_len, k_len):
        if case.get("causal", True):
            first = max(0, q - k)  # rows before it see nothing
            seen = q - first
            pairs += seen * k - seen * (seen - 1) // 2
        else:
            pairs += q * k
    read = (nq * hq + 2 * nk * hk) * dim * b
    if op == "decode":
        return {"bytes": read + nq * hq * (dim * b + 4), "flops": 4 * pairs * hq * dim}
    # Forward two products, backward five (the scores are computed again).
    return {"bytes": 2 * read + nq * hq * (2 * dim * b + 4), "flops": 14 * pairs * hq * dim}


# The definitions in 64 bits.


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        return _exact_embed(s)
    if op in ("attend", "decode"):
        return _exact_attention(s)
    return _exact_loss(s)


def _exact_loss(s):
    case, tokens = s["case"], s["tokens"]
    n, vocab, temp = tokens.numel(), case["vocab"], case["temperature"]
    offsets = s["offsets"].tolist()
    on = tokens >= 0
    logp = torch.zeros(n, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 27) // vocab)
    for a in range(0, n, step):
        z = torch.log_softmax(s["logits"][a:a + step].double() / temp, 1)
        logp[a:a + step] = z.gather(1, tokens[a:a + step].clamp(min=0)[:, None])[:, 0]
    logp[~on] = 0
    ref = s["ref_logp"].double()
    coef = torch.zeros_like(logp)
    counts = [int(c) for c in torch.stack([on[a:b].sum() for a, b in zip(offsets, offsets[1:])])]
    got = {}
    if case["op"] == "policy":
        losses = torch.zeros_like(logp)
        for g in range(case["groups"]):
            ids = range(g * case["samples"], (g + 1) * case["samples"])
            m = torch.tensor([min(int(x), int(s["limits"][g])) for x in
                              s["makespans"][ids.start:ids.stop].tolist()], dtype=torch.float64)
            std = float(m.std(correction=0))
            adv = (m.mean() - m) / std if m.min() != m.max() else torch.zeros_like(m)
            for i, a_s in zip(ids, adv.tolist()):
                if not counts[i]:
                    continue
                w = 1.0 / sum(counts) if case["mean"] == "tokens" else \
                    1.0 / (counts[i] * sum(c > 0 for c in counts))
                at = torch.arange(offsets[i], offsets[i + 1], device="cuda")
                at = at[on[at]]
                r = torch.exp(logp[at] - s["old_logp"][at].double())
                bounded = torch.clamp(r, 1 - 0.2, 1 + 0.25)
                better = torch.minimum(r * a_s, bounded * a_s)
                x = ref[at] - logp[at]
                losses[at] = w * (0.04 * (torch.expm1(x) - x) - better)
                moves = (r * a_s <= bounded * a_s).double()
                coef[at] = w * (-0.04 * torch.expm1(x) - moves * a_s * r)
        got = {"loss": losses.sum().view(1), "losses": losses, "logp": logp}
    else:
        margins, loss, eps = [], 0.0, case["smoothing"]
        gain = torch.where(on, logp - ref, 0.0)
        for i in range(case["pairs"]):
            a, b, c = offsets[2 * i:2 * i + 3]
            m = 0.1 * float(gain[a:b].sum() - gain[b:c].sum())
            sig = 1 / (1 + math.exp(-m)) if m > -700 else 0.0
            loss -= ((1 - eps) * math.log(sig) + eps * math.log1p(-sig)) / case["pairs"]
            slope = 0.1 * (eps - (1 - sig)) / case["pairs"]
            coef[a:b], coef[b:c] = slope, -slope
            margins.append(m)
        coef[~on] = 0
        got = {"loss": torch.tensor([loss], dtype=torch.float64, device="cuda"),
               "margins": torch.tensor(margins, dtype=torch.float64, device="cuda"),
               "logp": logp, "d_logp": coef}
    d = torch.empty((n, vocab), dtype=torch.float64, device="cuda")
    for a in range(0, n, step):
        z = torch.softmax(s["logits"][a:a + step].double() / temp, 1).neg_()
        t = tokens[a:a + step].clamp(min=0)[:, None]
        z.scatter_add_(1, t, torch.ones_like(t, dtype=torch.float64))
        d[a:a + step] = z * (coef[a:a + step, None] / temp)
    got["d_logits"] = d
    return got


def _exact_embed(s):
    tokens, vocab = s["tokens"], s["table"].shape[0]
    rows = torch.zeros(s["d_rows"].shape, dtype=torch.float64, device="cuda")
    at = (tokens >= 0).nonzero()[:, 0]
    rows[at] = s["table"][tokens[at]].double() * s["scale"]
    d = torch.zeros((vocab, rows.shape[1]), dtype=torch.float64, device="cuda")
    order = tokens[at].argsort()
    names, counts = torch.unique_consecutive(tokens[at][order], return_counts=True)
    ends = counts.cumsum(0).tolist()
    step = max(1, (1 << 26) // rows.shape[1])
    # Whole runs of equal tokens at a time; a run's sum is taken as one product.
    start = run = 0
    for i, end in enumerate(ends):
        if i + 1 < len(ends) and ends[i + 1] - start <= step:
            continue
        part = s["d_rows"][at[order[start:end]]].double()
        which = torch.repeat_interleave(torch.arange(i + 1 - run, device="cuda"), counts[run:i + 1])
        d.index_put_((names[run:i + 1],), torch.zeros((i + 1 - run, rows.shape[1]),
                     dtype=torch.float64, device="cuda").index_add_(0, which, part) * s["scale"])
        start, run = end, i + 1
    if "acc" in s:
        d += s["acc"].double()
    return {"rows": rows, "d_table": d}


def _exact_attention(s):
    case = s["case"]
    q_at, k_at = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    shape = {"out": s["q"], "d_q": s["q"], "d_k": s["k"], "d_v": s["v"]}
    got = {n: torch.zeros(x.shape, dtype=torch.float64, device="cuda") for n, x in shape.items()
           if n == "out" or case["op"] == "attend"}
    got["lse"] = torch.full((hq, s["q"].shape[0]), -math.inf, dtype=torch.float64, device="cuda")
    lengths = s["k_lengths"].tolist() if "k_lengths" in s else \
        [b - a for a, b in zip(k_at, k_at[1:])]
    for b in range(case["batch"]):
        rq = slice(q_at[b], q_at[b + 1])
        rk = slice(k_at[b], k_at[b] + lengths[b])
        nq, nk = rq.stop - rq.start, lengths[b]
        if not nq or not nk:
            continue
        for h in range(hq):
            g = h // (hq // hk)
            q, k, v = s["q"][rq, h].double(), s["k"][rk, g].double(), s["v"][rk, g].double()
            a = q @ k.T / math.sqrt(dim)
            if case.get("causal", True):
                last = torch.arange(nq, device="cuda")[:, None] + (nk - nq)
                a[torch.arange(nk, device="cuda")[None] > last] = -math.inf
            lse = torch.logsumexp(a, 1, keepdim=True)
            p = torch.where(lse == -math.inf, 0.0, torch.exp(a - lse))
            out = p @ v
            got["out"][rq, h], got["lse"][h, rq] = out, lse[:, 0]
            if case["op"] == "attend":
                do = s["d_out"][rq, h].double()
                got["d_v"][rk, g] += p.T @ do
                ds = p * (do @ v.T - (do * out).sum(1, keepdim=True)) / math.sqrt(dim)
                got["d_q"][rq, h] = ds @ k
                got["d_k"][rk, g] += ds.T @ q
    return got
