"""Plain 64-bit forms of the operators of include/sched_policy.h on the CPU,
with bounds on what a kernel may differ by.

A bound adds up, element by element, the roundings that the operator's
definition allows: U of the type for each rounding to it (its products' 16-bit
operands, its result), 2^-24 for every 32-bit step.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -140, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -130}
F = 2.0 ** -24
LEAST = 2.0 ** -126  # probabilities below it count as zero


def f32(x):
    """A factor as the calls take it, in 32 bits."""
    return torch.tensor(x, dtype=torch.float32).double().item()


def close(got, want, bound, what=""):
    """Element by element; infinities and NaN have to be the same."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.nan_to_num(got[odd], 7e77), torch.nan_to_num(want[odd], 7e77)), what
    off = (got - want)[~odd].abs()
    most = torch.as_tensor(bound, dtype=torch.float64).expand(want.shape)[~odd]
    assert bool((off <= most).all()), (what, float((off - most).max()), float((off / most).max()))


def embed(table, tokens, scale):
    on = (tokens >= 0) & (tokens < table.shape[0])
    rows = torch.zeros((tokens.numel(), table.shape[1]), dtype=torch.float64)
    rows[on] = table.double()[tokens[on].long()] * scale
    return rows


def embed_grad(d_rows, tokens, vocab, scale):
    """(gradient, sum of magnitudes, most rows of a token)."""
    d = torch.zeros((vocab, d_rows.shape[1]), dtype=torch.float64)
    size = torch.zeros_like(d)
    count = torch.zeros(vocab, dtype=torch.float64)
    for i, t in enumerate(tokens.tolist()):
        if 0 <= t < vocab:
            d[t] += d_rows[i].double() * scale
            size[t] += (d_rows[i].double() * scale).abs()
            count[t] += 1
    return d, size, count


def logprobs(logits, tokens, temperature):
    """(log-probabilities, probabilities, rows with a loss)."""
    z = logits.double() / f32(temperature)
    on = (tokens >= 0) & (tokens < logits.shape[1])
    most = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isfinite(most), most, 0.0))
    total = e.sum(1, keepdim=True)
    t = torch.where(on, tokens, 0).long()[:, None]
    logp = (z.gather(1, t) - torch.where(torch.isfinite(most), most, 0.0) - torch.log(total))[:, 0]
    logp = torch.where(total[:, 0] == 0, -math.inf, logp)
    p = e / total
    return torch.where(on, logp, 0.0), torch.where(p < LEAST, 0.0, p), on


def logits_error(logits, temperature):
    """Relative error of a probability in 32 bits, per row: every exponent is a
    difference rounded, times a rounded factor, to a power of 1 ulp; the sum
    adds a term per rounding."""
    z = logits.double() / temperature
    z = torch.where(torch.isfinite(z) & (z.abs() < 1e30), z, 0.0)
    span = z.amax(1) - z.amin(1) + z.abs().amax(1)
    return F * (8 * span + logits.shape[1] / 64 + 64)


def d_logits(logits, tokens, p, on, logp, d_logp, temperature):
    g = torch.where(on & (logp > -math.inf), d_logp.double(), 0.0)[:, None] / temperature
    hot = torch.zeros_like(p)
    hot[torch.arange(len(tokens)), torch.where(on, tokens, 0).long()] = 1
    want = torch.where(g == 0, 0.0, g * (hot - p))
    p = torch.nan_to_num(p)
    err = logits_error(logits, temperature)[:, None]
    bound = g.abs() * (2 * err * p + 4 * F) + U[logits.dtype] * want.abs() + TINY[logits.dtype]
    return want, bound


def policy(logp, on, old, ref, adv, weights, lo, hi, kl):
    """(losses, derivative by logp)."""
    lo, hi, kl = f32(lo), f32(hi), f32(kl)
    r = torch.exp(logp - old.double())
    a, w = adv.double(), weights.double()
    free, held = -a * r, -a * r.clamp(1 - lo, 1 + hi)
    loss, slope = torch.maximum(free, held), torch.where(free >= held, free, 0.0)
    if kl:
        e = ref.double() - logp
        loss, slope = loss + kl * (torch.exp(e) - e - 1), slope + kl * (1 - torch.exp(e))
    return torch.where(on, w * loss, 0.0), torch.where(on, w * slope, 0.0)


def advantages(makespans, limits, groups, offsets, tokens, mean):
    adv = torch.zeros(len(tokens), dtype=torch.float64)
    weight = torch.zeros(len(tokens), dtype=torch.float64)
    n = len(makespans)
    counts = [int((tokens[offsets[i]:offsets[i + 1]] >= 0).sum()) for i in range(n)]
    for g in range(len(limits)):
        m = [min(int(x), int(limits[g])) for x in makespans[groups[g]:groups[g + 1]]]
        for i in range(groups[g], groups[g + 1]):
            mid = sum(m) / len(m)
            dev = math.sqrt(sum((x - mid) ** 2 for x in m) / len(m))
            at = slice(offsets[i], offsets[i + 1])
            adv[at] = (mid - m[i - groups[g]]) / dev if min(m) < max(m) else 0.0
            if counts[i]:
                total = sum(counts) if mean == "tokens" else counts[i] * sum(c > 0 for c in counts)
                weight[at] = (tokens[at] >= 0).double() / total
    return adv, weight


def preference(logp, ref, tokens, offsets, beta, eps):
    beta, eps = f32(beta), f32(eps)
    pairs = (len(offsets) - 1) // 2
    on = tokens >= 0
    gain = torch.where(on, logp.double() - ref.double(), 0.0)
    margins, d = torch.zeros(pairs, dtype=torch.float64), torch.zeros_like(gain)
    for p in range(pairs):
        a, b, c = offsets[2 * p:2 * p + 3]
        m = margins[p] = beta * (gain[a:b].sum() - gain[b:c].sum())
        slope = beta * (eps * torch.sigmoid(m) - (1 - eps) * torch.sigmoid(-m)) / pairs
        d[a:b], d[b:c] = slope, -slope
    loss = -(1 - eps) * torch.nn.functional.logsigmoid(margins) - \
        eps * torch.nn.functional.logsigmoid(-margins)
    return loss.mean(), margins, torch.where(on, d, 0.0)


class Attention:
    """Forward and backward of one call, sequence by sequence and head by head,
    and the bounds of every result."""

    def __init__(self, q, k, v, q_off, k_off, k_len, causal, scale, d_out=None):
        scale = f32(scale)
        t = q.dtype
        u, tiny = U[t], TINY[t]
        q, k, v = q.double(), k.double(), v.double()
        rows, heads, dim = q.shape
        group = heads // k.shape[1]
        zeros = lambda x: torch.zeros_like(x)  # noqa: E731
        self.out, self.out_b = zeros(q), zeros(q)
        self.lse = torch.full((heads, rows), -math.inf, dtype=torch.float64)
        self.lse_b = torch.zeros((heads, rows), dtype=torch.float64)
        self.dq, self.dk, self.dv = zeros(q), zeros(k), zeros(v)
        self.dq_b, self.dk_b, self.dv_b = zeros(q), zeros(k), zeros(v)
        for b in range(len(q_off) - 1):
            n = k_off[b + 1] - k_off[b] if k_len is None else k_len[b]
            rq, rk = slice(q_off[b], q_off[b + 1]), slice(k_off[b], k_off[b] + n)
            m = rq.stop - rq.start
            if m <= 0 or n <= 0:
                continue
            seen = torch.ones((m, n), dtype=torch.bool)
            if causal:
                seen = torch.arange(n)[None] <= torch.arange(m)[:, None] + (n - m)
            for h in range(heads):
                g = h // group
                Q, K, V = q[rq, h], k[rk, g], v[rk, g]
                s = (Q @ K.T * scale).masked_fill(~seen, -math.inf)
                lse = torch.logsumexp(s, 1, keepdim=True)
                P = torch.where(seen, torch.exp(s - lse), 0.0)
                P = torch.where(P < LEAST, 0.0, torch.nan_to_num(P))
                out = P @ V
                # A score's error: D + 8 roundings of terms of its products, and
                # those of the exponent and the sum.
                size = s.nan_to_num(0, 0, 0).abs()
                ds = F * ((dim + 16) * (Q.abs() @ K.abs().T * scale) + 4 * size + n / 16 + 64)
                ds = 2 * ds.amax(1, keepdim=True)
                self.out[rq, h], self.lse[h, rq] = out, lse[:, 0]
                self.out_b[rq, h] = (u + ds) * (P @ V.abs()) + u * out.abs()
                self.out_b[rq, h] += tiny * (1 + n * V.abs().amax())
                self.lse_b[h, rq] = ds[:, 0] + 4 * F * lse[:, 0].nan_to_num(0, 0, 0).abs()
                if d_out is None:
                    continue
                dO = d_out[rq, h].double()
                self.dv[rk, g] += P.T @ dO
                # Probabilities from lse carry its error too.
                dp = 2 * ds + 4 * F * lse.nan_to_num(0, 0, 0).abs()
                self.dv_b[rk, g] += ((P * (u + dp)).T @ dO.abs()) + tiny * m * dO.abs().amax()
                dP, delta = dO @ V.T, (dO * out).sum(1, keepdim=True)
                dS = P * (dP - delta)
                # delta comes from the rounded out.
                d_err = (dO.abs() * self.out_b[rq, h]).sum(1, keepdim=True)
                s_err = P * (dp * (dP - delta).abs() + F * (dim + 16) * (dO.abs() @ V.abs().T)
                             + d_err + F * delta.abs()) + u * dS.abs() + tiny
                self.dq[rq, h] = dS @ K * scale
                self.dk[rk, g] += dS.T @ Q * scale
                self.dq_b[rq, h] = (s_err + F * n * dS.abs()) @ K.abs() * scale
                self.dk_b[rk, g] += (s_err + F * (m + 16) * dS.abs()).T @ Q.abs() * scale
                self.dv_b[rk, g] += F * (m + 16) * (P.T @ dO.abs())
        for x, y in ((self.dq_b, self.dq), (self.dk_b, self.dk), (self.dv_b, self.dv)):
            x += u * y.abs() + tiny
