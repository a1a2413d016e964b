"""The agent of workloads/agent.py with one prompt for many answers: the operators
together, as they are used."""
import itertools

import pytest
import torch

import paper_2607_22242_amd as S
from workloads import agent as A
from workloads import synth

pytestmark = pytest.mark.gpu


def relative(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("rotate", [False, True])
def test_a_shared_prompt_is_a_repeated_one(rotate):
    """Logits and gradients of the two packed passes, and logits over the caches,
    differ by the roundings of 16-bit attention: two layers' heads, rounded to 8
    bits once or twice on either side; gradients through both layers and back."""
    torch.manual_seed(1)
    flow = A.Workflow(synth.load(1), 9)
    model = A.Agent(flow.length, rotate=rotate).cuda()
    if rotate:
        with torch.no_grad():
            for w in (model.q_norms, model.k_norms):
                w.mul_(1 + 0.2 * torch.randn_like(w))
    modes, cached = A.sample_shared(model, flow)
    d = torch.randn(9 * flow.n, A.MODES, device="cuda")
    got = []
    for shared in (False, True):
        model.zero_grad()
        logits = flow.logits(model, modes, shared)
        logits.backward(d)
        got.append((logits.detach(), [p.grad for p in model.parameters() if p.grad is not None]))
    u = 2.0 ** -8
    assert relative(got[1][0], got[0][0]) < 2 * 2 * u
    assert relative(cached.reshape(-1, A.MODES), got[0][0]) < 2 * 2 * u
    assert len(got[0][1]) == len(got[1][1])
    for a, b in zip(got[1][1], got[0][1]):
        assert relative(a, b) < 4 * 2 * 2 * u


@pytest.mark.parametrize("rotate", [False, True])
def test_single_tokens_see_what_the_packed_pass_does(rotate):
    torch.manual_seed(3)
    flow = A.Workflow(synth.load(0), 5)
    model = A.Agent(flow.length, rotate=rotate).cuda()
    modes, cached = A.sample(model, flow)
    with torch.no_grad():
        packed = flow.logits(model, modes)
    assert relative(cached.reshape(-1, A.MODES), packed) < 2 * 2 * 2.0 ** -8


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_gradient_of_the_whole_step(loss):
    """A step's gradient against the loss's own differences along it."""
    torch.manual_seed(2)
    flow = A.Workflow(synth.load(0), 8)
    model = A.Agent(flow.length, rotate=True).cuda()
    modes, logits = A.sample_shared(model, flow)
    old = S.sched_token_logprobs(logits.reshape(-1, A.MODES), modes.reshape(-1)) - 0.05
    makespans = flow.makespans(modes)

    class Keep:  # in place of an optimizer
        def zero_grad(self):
            model.zero_grad()

        def step(self):
            pass

    def value():
        return float(A.step(model, flow, Keep(), modes, old, old, makespans, loss, shared=True))

    value()
    params = [p for p in model.parameters() if p.grad is not None]
    grads = [p.grad.clone() for p in params]
    size = float(torch.sqrt(sum(g.square().sum() for g in grads)))
    values = []
    h = 0.02 / size
    for sign in (1, -1):
        with torch.no_grad():
            for p, g in zip(params, grads):
                p.add_(g, alpha=sign * h)
        values.append(value())
        with torch.no_grad():
            for p, g in zip(params, grads):
                p.sub_(g, alpha=sign * h)
    slope = (values[0] - values[1]) / (2 * h)
    # Along the gradient the slope is its squared length; 16-bit attention moves
    # either loss by some 2^-9 of its terms, which the step of 0.02 divides.
    assert abs(slope - size ** 2) < 0.15 * size ** 2


def test_beams_of_every_mapping():
    """As many beams as there are mappings of four tools: all of them, in the order
    of their log-probabilities by the packed pass."""
    inst = synth.load(0)  # a chain, of which the first four tools
    flow = A.Workflow(dict(inst, tools=inst["tools"][:4], edges=inst["edges"][:3], n_tools=4), 81)
    torch.manual_seed(5)
    model = A.Agent(flow.length, rotate=True).cuda()
    with torch.no_grad():
        model.head.mul_(4)  # mappings apart from one another
        every = torch.tensor(list(itertools.product(range(A.MODES), repeat=4)), device="cuda")
        logp = torch.log_softmax(flow.logits(model, every, shared=True).double(), 1)
        total = logp.gather(1, every.reshape(-1, 1)).view(81, 4).sum(1)
    modes, scores = A.beams(model, flow, 81)
    assert len(modes) == 81 and len({tuple(m) for m in modes.tolist()}) == 81
    assert bool((scores[:-1] >= scores[1:]).all())
    names = {tuple(m): i for i, m in enumerate(every.tolist())}
    order = torch.tensor([names[tuple(m)] for m in modes.tolist()], device="cuda")
    # Logits are within 2 2 2^-8 of the packed pass's in norm, four of them add up.
    size = float(torch.log_softmax(logp, 1).abs().max())
    assert float((scores.double() - total[order]).abs().max()) < 4 * 2 * 2 * 2.0 ** -8 * max(size, 4.0)
    # Fewer beams keep the best of what they meet, and no mapping twice.
    few, best = A.beams(model, flow, 7)
    assert len(few) == 7 and len({tuple(m) for m in few.tolist()}) == 7
    found = total[torch.tensor([names[tuple(m)] for m in few.tolist()], device="cuda")]
    assert float((best.double() - found).abs().max()) < 4 * 2 * 2 * 2.0 ** -8 * max(size, 4.0)


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_training_runs(loss):
    means, best, flow = A.train(synth.load(1), rounds=3, samples=32, loss=loss, shared=True, rotate=True, width=40)
    assert len(means) == 3 and best >= flow.optimum()


def test_a_second_derivative_is_refused():
    x = torch.randn(5, 4, 16, device="cuda").bfloat16().requires_grad_()
    ends = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    w, places = torch.ones(16, device="cuda"), torch.arange(5, device="cuda")
    for out in (A.AttendShared.apply(x, x, 2, ends, ends, one),
                A.NormRotate.apply(x, 2, w, w, places, torch.ones(8, device="cuda"))):
        d, = torch.autograd.grad(out.float().square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="differentiat"):
            d.float().square().sum().backward()
