"""A small agent that answers with device mappings and learns from the search's
scores (Section 3.3 has a language model answer; here a transformer of a few
layers stands for it, so that a run takes seconds).

The prompt is the tool cards of a workflow as bucketed tokens, the answer one
mode token per tool.  A round samples answers over a key/value cache
(sched_attention of single tokens), scores them as mappings
(sched_eval_mappings_device), turns their makespans into advantages
(sched_group_advantages) and takes a step on the clipped policy loss
(sched_policy_loss), or on the preference loss over pairs of a better and a
worse answer (sched_token_logprobs, sched_preference_loss), through attention
and the embedding (sched_attention_grad, sched_embed_grad).  Dense products
are the library's, norms torch's.

    python -m workloads.agent [--config 0..3] [--rounds 60] [--samples 128]
                              [--loss policy|preference]

prints a line per ten rounds: the mean makespan of the round's answers and the
best one so far, then the optimum that the search finds.  On the 12-tool
workload (3^12 mappings) the answers end at the optimum, on the 16-tool one
within some per cent of it, after a few thousand scored answers.
"""
from __future__ import annotations

import argparse
import math

import torch
from torch.autograd.function import once_differentiable

import paper_2607_22242_amd as S
from workloads import synth

MODES, BUCKETS, FIELDS = 3, 24, 5
START = MODES + FIELDS * BUCKETS  # the token behind the cards
VOCAB = START + 1


def prompt(inst):
    """Tokens of the tool cards (the octave of each field) and the start."""
    out = []
    for tool in inst["tools"]:
        for f, x in enumerate(tool):
            bucket = min(BUCKETS - 1, int(math.log2(x + 1)))
            out.append(MODES + f * BUCKETS + bucket)
    return out + [START]


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, tokens, scale):
        ctx.save_for_backward(tokens)
        ctx.vocab, ctx.scale = table.shape[0], scale
        return S.sched_embed(table, tokens, scale=scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, d_rows):
        tokens, = ctx.saved_tensors
        return S.sched_embed_grad(d_rows.contiguous(), tokens, ctx.vocab, scale=ctx.scale), None, None


class Attend(torch.autograd.Function):
    """Causal attention of packed sequences, q, k and v slices of one tensor."""

    @staticmethod
    def forward(ctx, x, heads, offsets):
        kv = (x.shape[1] - heads) // 2
        q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
        out, lse = S.sched_attention(q, k, v, offsets, offsets)
        ctx.save_for_backward(x, out, lse, offsets)
        ctx.heads = heads
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, d_out):
        x, out, lse, offsets = ctx.saved_tensors
        h, kv = ctx.heads, (x.shape[1] - ctx.heads) // 2
        d = torch.empty_like(x)
        S.sched_attention_grad(x[:, :h], x[:, h:h + kv], x[:, h + kv:], out, lse, d_out.contiguous(),
                               offsets, offsets, d_q=d[:, :h], d_k=d[:, h:h + kv], d_v=d[:, h + kv:])
        return d, None, None


class Agent(torch.nn.Module):
    def __init__(self, positions, width=128, heads=4, kv_heads=2, layers=2):
        super().__init__()
        self.width, self.heads, self.kv, self.dim = width, heads, kv_heads, width // heads
        new = lambda *shape: torch.nn.Parameter(torch.randn(shape) / math.sqrt(shape[0]))  # noqa: E731
        self.tokens = torch.nn.Parameter(torch.randn(VOCAB, width) / math.sqrt(width))
        self.places = torch.nn.Parameter(torch.randn(positions, width) / math.sqrt(width))
        self.blocks = torch.nn.ParameterList()
        for _ in range(layers):
            self.blocks.extend([new(width, (heads + 2 * kv_heads) * self.dim), new(width, width),
                                new(width, 4 * width), new(4 * width, width)])
        self.head = new(width, MODES)

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def run(self, tokens, places, attend):
        """Logits of the rows; attend(layer, x) maps q, k and v to the heads' outputs."""
        scale = math.sqrt(self.width)
        x = Embed.apply(self.tokens, tokens, scale) + Embed.apply(self.places, places, scale)
        for i in range(len(self.blocks) // 4):
            qkv, out, up, down = self.blocks[4 * i:4 * i + 4]
            y = (self.norm(x) @ qkv).bfloat16().view(len(x), -1, self.dim)
            x = x + attend(i, y).float().view(len(x), self.width) @ out
            x = x + torch.nn.functional.silu(self.norm(x) @ up) @ down
        return self.norm(x) @ self.head

    def packed(self, tokens, places, offsets):
        return self.run(tokens, places, lambda i, y: Attend.apply(y, self.heads, offsets))


class Workflow:
    """A problem, its prompt, and what scores answers of it."""

    def __init__(self, inst, samples, device="cuda"):
        self.problem = S.Problem.from_instance(inst)
        self.n, self.samples = self.problem.n, samples
        self.ws = S.workspace([self.problem.handle], device=device)
        self.prompt = torch.tensor(prompt(inst), device=device)
        self.length = len(self.prompt) + self.n  # the last answer is never read
        self.weights = 3 ** torch.arange(self.n, device=device)
        self.group = torch.tensor([0, samples], dtype=torch.int32, device=device)
        self.answers = torch.arange(samples + 1, dtype=torch.int32, device=device) * self.n
        self.all_cpu = int(S.sched_eval_mappings(self.problem.handle, [0], self.ws)[0])
        # An answer that runs out of memory counts as twice the all-CPU mapping.
        self.limit = torch.tensor([2 * self.all_cpu], device=device)

    def optimum(self):
        return S.sched_bruteforce_argmin(self.problem.handle, 0, self.problem.n_mappings, self.ws)[1]

    def makespans(self, modes):
        index = (modes * self.weights).sum(1)
        out = torch.empty_like(index)
        S.sched_eval_mappings_device(self.problem.handle, index, out, self.ws)
        return out

    def rows(self, modes):
        """(tokens, places, offsets, rows that predict an answer) of the packed
        sequences prompt + all but the last answer."""
        tokens = torch.cat([self.prompt.expand(self.samples, -1), modes[:, :-1]], 1)
        count = tokens.shape[1]
        places = torch.arange(count, device=tokens.device).expand_as(tokens)
        offsets = torch.arange(self.samples + 1, dtype=torch.int32, device=tokens.device) * count
        predict = places >= len(self.prompt) - 1
        return tokens.reshape(-1), places.reshape(-1), offsets, predict.reshape(-1)


@torch.no_grad()
def sample(agent, flow):
    """(modes, logits) of one answer per sample, over a cache of slots."""
    b, slot, device = flow.samples, flow.length, flow.prompt.device
    layers, h, kv = len(agent.blocks) // 4, agent.heads, agent.kv
    cache = torch.empty((layers, 2, b, slot, kv, agent.dim), dtype=torch.bfloat16, device=device)
    k_offsets = torch.arange(b + 1, dtype=torch.int32, device=device) * slot
    lengths = torch.zeros(b, dtype=torch.int32, device=device)

    def attend(at, count):
        q_offsets = torch.arange(b + 1, dtype=torch.int32, device=device) * count

        def of_layer(i, y):
            y3 = y.view(b, count, -1, agent.dim)
            cache[i, 0, :, at:at + count], cache[i, 1, :, at:at + count] = \
                y3[:, :, h:h + kv], y3[:, :, h + kv:]
            k, v = (cache[i, j].view(b * slot, kv, agent.dim) for j in (0, 1))
            return S.sched_attention(y[:, :h], k, v, q_offsets, k_offsets, k_lengths=lengths)[0]
        return of_layer

    tokens, at = flow.prompt.repeat(b, 1), 0
    modes, all_logits = [], []
    for _ in range(flow.n):
        count = tokens.shape[1]
        lengths.fill_(at + count)
        places = torch.arange(at, at + count, device=device).repeat(b)
        logits = agent.run(tokens.reshape(-1), places, attend(at, count)).view(b, count, MODES)[:, -1]
        modes.append(torch.multinomial(torch.softmax(logits, 1), 1))
        all_logits.append(logits)
        tokens, at = modes[-1], at + count
    return torch.cat(modes, 1), torch.stack(all_logits, 1)


def step(agent, flow, optimizer, modes, old_logp, ref_logp, makespans, loss="policy", scale=1.0):
    """One update on the round's answers; returns the loss (on the device)."""
    tokens, places, offsets, predict = flow.rows(modes)
    logits = agent.packed(tokens, places, offsets)[predict]
    answers = modes.reshape(-1)
    if loss == "policy":
        adv, weights = S.sched_group_advantages(makespans, flow.limit, flow.group, flow.answers,
                                                answers)
        value, _, _, d_logits = S.sched_policy_loss(logits.detach(), answers, old_logp, ref_logp, adv,
                                                    weights, clip_low=0.2, clip_high=0.25,
                                                    kl_weight=0.01, loss_scale=scale)
    else:
        # Pairs: the best half against the worst half, best with worst.
        order = makespans.argsort()
        half = flow.samples // 2
        pairs = torch.stack([order[:half], order.flip(0)[:half]], 1).reshape(-1)
        at = (pairs[:, None] * flow.n + torch.arange(flow.n, device=pairs.device)).reshape(-1)
        chosen, tok, ref = logits.detach()[at], answers[at], ref_logp[at]
        logp = S.sched_token_logprobs(chosen, tok)
        value, _, d_logp = S.sched_preference_loss(logp, ref, tok, flow.answers[:2 * half + 1],
                                                   beta=0.1, loss_scale=scale)
        d_logits = torch.zeros_like(logits)
        d_logits[at] = S.sched_token_logprobs_grad(chosen, tok, logp, d_logp, d_logits=chosen)
    optimizer.zero_grad()
    logits.backward(d_logits)
    optimizer.step()
    return value


def train(inst, rounds=60, samples=128, loss="policy", seed=0, lr=5e-4, tell=None):
    """Mean makespans of the rounds' answers (limited), and the best one found."""
    torch.manual_seed(seed)
    flow = Workflow(inst, samples)
    agent = Agent(flow.length).cuda()
    optimizer = torch.optim.Adam(agent.parameters(), lr=lr)
    means, best = [], 2 * flow.all_cpu
    for r in range(rounds):
        modes, logits = sample(agent, flow)
        makespans = flow.makespans(modes)
        old = S.sched_token_logprobs(logits.view(-1, MODES), modes.reshape(-1))
        for _ in range(2):
            step(agent, flow, optimizer, modes, old, old, makespans, loss)
        means.append(float(torch.minimum(makespans, flow.limit).double().mean()))
        best = min(best, int(makespans.min()))
        if tell is not None and r % 10 == 9:
            tell(f"round {r + 1}: mean makespan {means[-1] / 1e3:.1f} ms, best so far "
                 f"{best / 1e3:.1f} ms")
    return means, best, flow


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", type=int, default=1, choices=range(4))
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--samples", type=int, default=128)
    ap.add_argument("--loss", choices=("policy", "preference"), default="policy")
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    means, best, flow = train(synth.load(a.config), a.rounds, a.samples, a.loss, a.seed,
                              tell=lambda s: print(s, flush=True))
    print(f"first round's mean {means[0] / 1e3:.1f} ms, last round's {means[-1] / 1e3:.1f} ms, best "
          f"{best / 1e3:.1f} ms, optimum {flow.optimum() / 1e3:.1f} ms, all on the CPU "
          f"{flow.all_cpu / 1e3:.1f} ms")


if __name__ == "__main__":
    main()
