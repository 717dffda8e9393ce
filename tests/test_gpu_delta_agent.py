"""The agent with a matrix for its memory: its operators together, as they would be used, and the gradients of its losses against plain ones in 64 bits."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("delta_agent", os.path.join(ROOT, "examples", "delta_agent.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_runs(example):
    fitness, losses = example.main(rounds=3, configurations=64, steps=20, heads=4, key_dim=16, value_dim=16, verbose=False)
    assert len(fitness) == 3 and all(map(math.isfinite, fitness + losses)) and min(losses) > -1e-6


def plain_layer(q, k, v, g, beta):
    group = v.shape[2] // q.shape[2]
    q, k = q.repeat_interleave(group, 2), k.repeat_interleave(group, 2)
    s, out = torch.zeros(v.shape[0], v.shape[2], q.shape[3], v.shape[3], dtype=v.dtype, device=v.device), []
    for t in range(v.shape[1]):
        s = torch.exp(g[:, t])[:, :, None, None] * s
        y = v[:, t] - (s * k[:, t, :, :, None]).sum(2)
        s = s + k[:, t, :, :, None] * (beta[:, t, :, None] * y)[:, :, None]
        out.append(q.shape[3] ** -0.5 * (s * q[:, t, :, :, None]).sum(2))
    return torch.stack(out, 1), s


def plain_logprobs(logits, tokens):
    logp = torch.log_softmax(logits, 1)

    class Result:
        logprob, entropy = logp.gather(1, tokens.long()[:, None])[:, 0], -(logp.exp() * logp).sum(1)
    return Result


def plain_distill(logits, tokens, scores):
    logp = torch.log_softmax(scores.to(logits.dtype), 1)
    return ((logp.exp() * (logp - torch.log_softmax(logits, 1).gather(1, tokens.long()))).sum(1),)


def wide(agent):
    """The same agent in 64 bits."""
    other = object.__new__(type(agent))
    other.__dict__.update({n: x for n, x in agent.__dict__.items() if n != "optimizer"})
    other.params = [p.detach().double().requires_grad_() for p in agent.params]
    return other


@pytest.mark.parametrize("steps", [5, 40, 100])
def test_gradients(example, steps):
    """Losses are means over at most 24 x 100 x 8 rows; gradients of chains of fp32 products (layer, two heads, rows), 2^-14 of the largest entry: 1024
    roundings of 2^-24, where each of some 10 products in a row sums at most 100 steps of like size."""
    gen = torch.Generator().manual_seed(steps)
    agent = example.DeltaAgent(8, 4, 16, 24, gen)
    n = 24
    xs = (torch.rand(n, steps, 8, generator=gen) * 2 - 1).cuda()
    actions = torch.randint(0, 3, (n, steps, 8), generator=gen, dtype=torch.int32).cuda()
    with torch.no_grad():
        logits, _ = agent.forward(xs)
        logps = plain_logprobs(logits.reshape(-1, 3), actions.reshape(-1)).logprob.view(actions.shape).sum(-1) + 0.05 * torch.randn(n, steps, generator=gen).cuda()
    advantage, returns = torch.randn(n, steps, generator=gen).cuda(), torch.randn(n, steps, generator=gen).cuda()
    batch = (xs, actions, logps, None, None)
    tokens, scores = example.taught_by(example.DeltaAgent(8, 2, 8, 8, gen), xs)
    exact = wide(agent)
    batch64 = (xs.double(), actions, logps.double(), None, None)
    pairs = [(example.policy_loss(agent, batch, advantage, returns),
              example.policy_loss(exact, batch64, advantage.double(), returns.double(), plain_layer, plain_logprobs)),
             (example.teaching_loss(agent, xs, tokens, scores), example.teaching_loss(exact, xs.double(), tokens, scores, plain_layer, plain_distill))]
    for mine, plain in pairs:
        assert abs(float(mine.detach()) - float(plain.detach())) <= 2.0 ** -14 * (1 + abs(float(plain.detach())))
        got = torch.autograd.grad(mine, agent.params, allow_unused=True)
        want = torch.autograd.grad(plain, exact.params, allow_unused=True)
        for i, (x, y) in enumerate(zip(got, want)):
            assert (x is None) == (y is None)
            if x is not None:
                assert float((x.double() - y).abs().max()) <= 2.0 ** -14 * float(y.abs().max()), i
