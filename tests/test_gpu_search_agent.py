"""The example's search agent: rollout, advantages, training and sampling together on the library's operators."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("search_agent", os.path.join(ROOT, "examples", "search_agent.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("state_bits", [32, 8])
def test_the_agent_climbs(example, state_bits):
    """Forty rounds of 256 configurations: the last five end higher than the first five."""
    fitness, chosen = example.main(rounds=40, configurations=256, steps=24, width=32, state_bits=state_bits, verbose=False)
    assert sum(fitness[-5:]) > sum(fitness[:5])
    assert chosen.dtype == torch.int32 and chosen.shape[1] == 8 and (chosen >= 0).all()


def test_recurrence_inside_autograd(example):
    """The gradients that autograd gets equal those of the same layer written as a loop in fp64, to 64 roundings of the largest (50 steps, gates below 1)."""
    gen = torch.Generator().manual_seed(1)
    a = torch.sigmoid(torch.randn(3, 50, 7, generator=gen)).cuda().requires_grad_()
    b, h0 = torch.randn(3, 50, 7, generator=gen).cuda().requires_grad_(), torch.randn(3, 7, generator=gen).cuda().requires_grad_()
    weight = torch.randn(3, 50, 7, generator=gen).cuda()
    got = torch.autograd.grad((example.Scan.apply(a, b, h0) * weight).sum(), (a, b, h0))
    h, total = h0.double(), 0.0
    for t in range(50):
        h = a[:, t].double() * h + b[:, t].double()
        total = total + (h * weight[:, t].double()).sum()
    for x, y in zip(got, torch.autograd.grad(total, (a, b, h0))):
        assert (x.double() - y.double()).abs().max() <= 2.0 ** -18 * y.abs().max()
