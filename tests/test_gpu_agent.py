"""The agent of workloads/agent.py: the operators together, as they are used."""
import pytest
import torch

import paper_2607_22242_amd as S
from workloads import agent as A
from workloads import synth

pytestmark = pytest.mark.gpu


def test_cached_answers_have_the_packed_pass_s_logits():
    """Single tokens over the cache and the packed training pass see the same
    model: their logits differ by the roundings of 16-bit attention."""
    torch.manual_seed(1)
    flow = A.Workflow(synth.load(1), 9)
    model = A.Agent(flow.length).cuda()
    modes, logits = A.sample(model, flow)
    tokens, places, offsets, predict = flow.rows(modes)
    with torch.no_grad():
        packed = model.packed(tokens, places, offsets)[predict].view(9, flow.n, A.MODES)
    # Two layers' heads, rounded to 8 bits once or twice on either side.
    assert float((packed - logits).norm() / logits.norm()) < 2 * 2 * 2.0 ** -8


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_gradient_of_the_whole_step(loss):
    """A step's gradient against the loss's own differences along it."""
    torch.manual_seed(2)
    flow = A.Workflow(synth.load(0), 8)
    model = A.Agent(flow.length).cuda()
    modes, logits = A.sample(model, flow)
    old = S.sched_token_logprobs(logits.view(-1, A.MODES), modes.reshape(-1)) - 0.05
    makespans = flow.makespans(modes)

    class Keep:  # in place of an optimizer
        def zero_grad(self):
            model.zero_grad()

        def step(self):
            pass

    args = (flow, Keep(), modes, old, old, makespans, loss)
    A.step(model, *args)
    grads = [p.grad.clone() for p in model.parameters()]
    size = float(torch.sqrt(sum(g.square().sum() for g in grads)))
    values = []
    h = 0.02 / size
    for sign in (1, -1):
        with torch.no_grad():
            for p, g in zip(model.parameters(), grads):
                p.add_(g, alpha=sign * h)
        values.append(float(A.step(model, *args)))
        with torch.no_grad():
            for p, g in zip(model.parameters(), grads):
                p.sub_(g, alpha=sign * h)
    slope = (values[0] - values[1]) / (2 * h)
    # Along the gradient the slope is its squared length; 16-bit attention moves
    # either loss by some 2^-9 of its terms, which the step of 0.02 divides.
    assert abs(slope - size ** 2) < 0.15 * size ** 2


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_training_lowers_the_makespans(loss):
    means, best, flow = A.train(synth.load(1), rounds=40, loss=loss)
    optimum = flow.optimum()
    assert best >= optimum
    assert means[-1] - optimum < 0.6 * (means[0] - optimum)


def test_a_second_derivative_is_refused():
    """The operators' gradients are no functions of their own to differentiate:
    torch says so in place of taking them as constants."""
    table = torch.randn(9, 16, device="cuda", requires_grad=True)
    tokens = torch.tensor([1, 4, 4], device="cuda")
    rows = A.Embed.apply(table, tokens, 2.0)
    d, = torch.autograd.grad(rows.square().sum(), table, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiat"):
        d.square().sum().backward()
    x = torch.randn(5, 4, 16, device="cuda").bfloat16().requires_grad_()
    out = A.Attend.apply(x, 2, torch.tensor([0, 5], dtype=torch.int32, device="cuda"))
    d, = torch.autograd.grad(out.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiat"):
        d.float().square().sum().backward()
