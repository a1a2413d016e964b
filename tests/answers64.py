"""Plain 64-bit forms, on the CPU, of the operators of include/sched_policy.h
that serve many answers to one prompt, with bounds on what a kernel may differ
by: U of the type for each rounding to it, 2^-24 for every 32-bit step."""
import math

import torch

from policy64 import F, LEAST, TINY, U, f32


def pairs_of(dim, turned, interleaved):
    """(first, second) elements of the pairs."""
    j = torch.arange(turned // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + turned // 2)


def rotated(x, positions, frequencies, interleaved, back=False):
    """x (rows x heads x dim) turned, and the magnitudes that its terms had."""
    a, b = pairs_of(x.shape[2], 2 * len(frequencies), interleaved)
    angle = positions.double()[:, None] * frequencies.double()
    if back:
        angle = -angle
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y, size = x.clone(), x.abs()
    if len(frequencies):
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        both = x[..., a].abs() + x[..., b].abs()
        size[..., a], size[..., b] = both, both
    return y, size


class Rotate:
    """Forward and backward of one tensor's heads, and the bounds."""

    def __init__(self, x, positions, frequencies, weight, norm, eps, interleaved, d_out=None):
        t, dim = x.dtype, x.shape[2]
        x = x.double()
        w = torch.ones(dim, dtype=torch.float64) if weight is None else weight.double()
        r = (x.square().mean(-1, keepdim=True) + f32(eps)).rsqrt() if norm else torch.ones_like(x[..., :1])
        # A sum of dim squares, its root, two products; an angle to 3.2 + 8
        # steps (2^31 turns of one), its cosine to two, a product and a sum.
        e = F * (dim + 32)
        self.out, size = rotated(x * r * w, positions, frequencies, interleaved)
        self.out_b = e * size + U[t] * self.out.abs() + TINY[t]
        if d_out is None:
            return
        g, size = rotated(d_out.double(), positions, frequencies, interleaved, back=True)
        y = x * r
        n = x.shape[0] * x.shape[1]
        self.dw = (g * y).sum((0, 1))
        self.dw_b = ((e + F * (n + 64)) * size * y.abs()).sum((0, 1)) + F * self.dw.abs()
        if norm:
            u = g * w
            self.dx = r * (u - y * (u * y).mean(-1, keepdim=True))
            wide = (w.abs() * size * y.abs()).mean(-1, keepdim=True)
            self.dx_b = 2 * e * r * (w.abs() * size + 2 * y.abs() * wide)
        else:
            self.dx, self.dx_b = g, e * size
        self.dx_b += U[t] * self.dx.abs() + TINY[t]


def beam_candidates(logits, scores, beams, last, end, temperature):
    """Per group a list of (score, beam, token), best first, equal ones by beam
    and token."""
    z = logits.double() / f32(temperature)
    groups = []
    for g in range(logits.shape[0] // beams):
        found = []
        for b in range(beams):
            i = g * beams + b
            start = float(scores[i])
            if not math.isfinite(start):
                continue
            if last is not None and end >= 0 and int(last[i]) == end:
                found.append((start, b, end))
                continue
            row = z[i]
            if bool(torch.isnan(row).any()) or bool((row == math.inf).any()) or bool((row == -math.inf).all()):
                continue
            # Sums and differences as the definition has them: one number per row.
            base = start - (float(row.max()) + math.log(float(torch.exp(row - row.max()).sum())))
            found += [(base + x, b, t) for t, x in enumerate(row.tolist()) if x > -math.inf]
        found.sort(key=lambda c: (-c[0], c[1], c[2]))
        groups.append(found)
    return groups


def beam_results(groups, beams, width, stay):
    """(scores, parents, tokens) in the groups' slots."""
    out = []
    for g, found in enumerate(groups):
        best = [(s, g * beams + b, t) for s, b, t in found[:width]]
        none = (-math.inf, -1, -1)
        if stay:
            slots, rest, seen = [None] * width, [], set()
            for c in best:
                if c[1] in seen:
                    rest.append(c)
                else:
                    slots[c[1] - g * beams] = c
                    seen.add(c[1])
            best = [c if c is not None else (rest.pop(0) if rest else none) for c in slots]
        out += best + [none] * (width - len(best))
    s, p, t = zip(*out) if out else ((), (), ())
    return torch.tensor(s, dtype=torch.float64), torch.tensor(p), torch.tensor(t)


def apart(groups, width, gap):
    """No two of the groups' best (and the next) of different beams are closer."""
    for found in groups:
        for a, b in zip(found[:width], found[1:width + 1]):
            if a[1] != b[1] and a[0] - b[0] < gap:
                return False
    return True


def reordered(states, parents, beams, lengths):
    out = states.clone()
    for s, p in enumerate(parents.tolist()):
        if p >= 0 and p // beams == s // beams:
            n = states.shape[2] if lengths is None else max(0, int(lengths[p]))
            out[:, s, :n] = states[:, p, :n]
    return out


class Shared:
    """Attention over shared prefixes, sequence by sequence and head by head:
    results, gradients and the bounds of every one."""

    def __init__(self, q, k, v, pk, pv, q_off, k_off, p_off, groups, k_len, p_len, causal, scale, d_out=None):
        scale, t = f32(scale), q.dtype
        u, tiny = U[t], TINY[t]
        q, k, v, pk, pv = (x.double() for x in (q, k, v, pk, pv))
        rows, heads, dim = q.shape
        share = heads // k.shape[1]
        zeros = torch.zeros_like
        self.out, self.out_b = zeros(q), zeros(q)
        self.lse = torch.full((heads, rows), -math.inf, dtype=torch.float64)
        self.lse_b = torch.zeros((heads, rows), dtype=torch.float64)
        self.dq, self.dk, self.dv, self.dpk, self.dpv = map(zeros, (q, k, v, pk, pv))
        self.dq_b, self.dk_b, self.dv_b, self.dpk_b, self.dpv_b = map(zeros, (q, k, v, pk, pv))
        of = {b: g for g in range(len(groups) - 1) for b in range(groups[g], groups[g + 1])}
        for b in range(len(q_off) - 1):
            g = of[b]
            own = k_off[b + 1] - k_off[b] if k_len is None else k_len[b]
            pre = p_off[g + 1] - p_off[g] if p_len is None else p_len[g]
            # Rows that a prefix key's sums run over.
            all_rows = (q_off[groups[g + 1]] - q_off[groups[g]]) * share
            rq, rk, rp = slice(q_off[b], q_off[b + 1]), slice(k_off[b], k_off[b] + own), slice(p_off[g], p_off[g] + pre)
            m, n = rq.stop - rq.start, own + pre
            if m <= 0 or n <= 0:
                continue
            seen = torch.ones((m, n), dtype=torch.bool)
            if causal:
                seen[:, pre:] = torch.arange(own)[None] <= torch.arange(m)[:, None] + (own - m)
            for h in range(heads):
                j = h // share
                Q, K, V = q[rq, h], torch.cat([pk[rp, j], k[rk, j]]), torch.cat([pv[rp, j], v[rk, j]])
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
                dp = 2 * ds + 4 * F * lse.nan_to_num(0, 0, 0).abs()  # probabilities from lse
                dv = P.T @ dO
                dv_b = ((P * (u + dp)).T @ dO.abs()) + F * (all_rows + 16) * (P.T @ dO.abs()) + \
                    tiny * m * dO.abs().amax()
                dP, delta = dO @ V.T, (dO * out).sum(1, keepdim=True)
                dS = P * (dP - delta)
                d_err = (dO.abs() * self.out_b[rq, h]).sum(1, keepdim=True)  # from the rounded out
                s_err = P * (dp * (dP - delta).abs() + F * (dim + 16) * (dO.abs() @ V.abs().T)
                             + d_err + F * delta.abs()) + u * dS.abs() + tiny
                self.dq[rq, h] = dS @ K * scale
                self.dq_b[rq, h] = (s_err + F * n * dS.abs()) @ K.abs() * scale
                dk = dS.T @ Q * scale
                dk_b = (s_err + F * (all_rows + 16) * dS.abs()).T @ Q.abs() * scale
                for x, part in ((self.dv, dv), (self.dv_b, dv_b), (self.dk, dk), (self.dk_b, dk_b)):
                    x[rk, j] += part[pre:]
                for x, part in ((self.dpv, dv), (self.dpv_b, dv_b), (self.dpk, dk), (self.dpk_b, dk_b)):
                    x[rp, j] += part[:pre]
        for x, y in ((self.dq_b, self.dq), (self.dk_b, self.dk), (self.dv_b, self.dv), (self.dpk_b, self.dpk),
                     (self.dpv_b, self.dpv)):
            x += u * y.abs() + tiny
