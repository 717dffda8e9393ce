"""Long rows whose cut falls among many entries that lie close together or are equal: draws as the definition has them.

A cut between distances that differ in fp32 is exact in any evaluation that orders alike, so the reference counts entries: whole numbers, fp32 distances and
weights of exp(d) in multiples of 2^-38 in fp64.  An fp32 exponential is off by 2^-22 of itself at most, so sums of weights are off by that, and the token
is one the reference draws for some number within 2^-21 and some p within 2^-21."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

EDGE = 2.0 ** -21


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def allowed(x, temperature, p, k, u):
    """First and last token of those that numbers and p within EDGE draw, and log-probabilities of both."""
    d = (x - x.max()) * (np.float32(1.0) / np.float32(temperature))
    order = np.argsort(-d, kind="stable")
    w = np.rint(np.exp(d.astype(np.float64)) * 2.0 ** 38)
    out = []
    for side in (-1, 1):
        kept = np.zeros(len(x))
        ws = w[order].copy()
        ws[k:] = 0
        before = np.cumsum(ws) - ws
        ws[1:][before[1:] >= p * (1 + side * EDGE) * ws.sum()] = 0
        kept[order] = ws
        total = kept.sum()
        run = np.cumsum(kept)
        for shift in (-EDGE, EDGE):
            token = int(np.searchsorted(run, max(u + shift, 0.0) * total, side="right"))
            token = min(token, int(np.flatnonzero(kept)[-1]))
            out.append((token, d[token] - np.log(total * 2.0 ** -38)))
    return out


ROWS = {
    "ordinary": lambda n, gen: torch.randn(n, generator=gen) * 2.0,
    "narrow with one far above": lambda n, gen: torch.cat([torch.tensor([9.0]), torch.randn(n - 1, generator=gen) * 0.01]),
    "few values": lambda n, gen: torch.randint(0, 40, (n,), generator=gen).float() * 0.25,
    "equal": lambda n, gen: torch.full((n,), 1.5),
}


@pytest.mark.parametrize("n", [60001, 262144, 1300007])
@pytest.mark.parametrize("kind", list(ROWS))
@pytest.mark.parametrize("temperature,p,k", [(1.25, 0.95, None), (1.0, 0.5, None), (1.5, 1.0, 20000), (0.7, 0.9, 50000)])
def test_crowded_cuts(rls, n, kind, temperature, p, k):
    gen = torch.Generator().manual_seed(n)
    row = ROWS[kind](n, gen)
    us = [0.0, 0.3, 0.77, 1.0 - 2.0 ** -24]
    logits = row[None].repeat(len(us), 1).cuda()
    fill = lambda v, t=torch.float32: torch.full((len(us),), v, dtype=t).cuda()      # noqa: E731
    token, logprob = rls.sample(logits, torch.tensor(us).cuda(), temperature=fill(temperature), top_p=fill(p) if p < 1 else None,
                                top_k=None if k is None else fill(k, torch.int32))
    x = row.numpy()
    for r, u in enumerate(us):
        some = allowed(x, temperature, p, n if k is None else k, float(np.float32(u)))
        tokens = [t for t, _ in some]
        assert min(tokens) <= token[r].item() <= max(tokens), (u, some, token[r])
        assert min(abs(lp - (logprob[r].item())) for _, lp in some) <= 2.0 ** -17 + 2.0 ** -20 * abs(logprob[r].item()) or min(tokens) < max(tokens)


def test_ordinary_logits_of_the_longest_rows(rls):
    """16,777,216 and 8,388,608 logits, temperatures above 1: the cut's bin holds some 20,000 to 40,000 of them."""
    gen = torch.Generator().manual_seed(5)
    row = torch.randn(1 << 24, generator=gen) * 2.0
    for n, temperature, p in ((1 << 23, 1.25, 0.95), (1 << 24, 1.5, 0.9)):
        x = row[:n]
        u = torch.tensor([0.6])
        token, _ = rls.sample(x[None].cuda(), u.cuda(), temperature=torch.tensor([temperature]).cuda(), top_p=torch.tensor([p]).cuda())
        some = [t for t, _ in allowed(x.numpy(), temperature, p, n, float(u))]
        assert min(some) <= token.item() <= max(some)
