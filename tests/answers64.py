"""Plain 64-bit forms, on the CPU, of the operators of include/sched_policy.h
that serve many answers to one prompt, with bounds on what a kernel may differ
by: U of the type for each rounding to it, 2^-24 for every 32-bit step."""
import math

import torch

from policy64 import F, TINY, U, f32


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
