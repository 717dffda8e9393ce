"""The first entry of a row's order where distances come together: it is drawn alone by top_k = 1, at every length of rows.

The order is by d = (x - max) * (1 / temperature) in fp32, equal ones by index: a large temperature makes neighbours equal that the logits tell apart."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

LENGTHS = [5, 20, 50, 100, 900, 12000, 30000, 140001]


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def first_of_the_order(row, temperature):
    x = row.numpy()
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        d = (x.max() - x) * (np.float32(1.0) / np.float32(temperature))
    d = np.where(np.isnan(d) | np.isinf(x), np.inf, d)
    return int(np.argmin(d))


@pytest.mark.parametrize("n", LENGTHS)
def test_top_k_of_one(rls, n):
    gen = torch.Generator().manual_seed(n)
    rows = [torch.randn(n, generator=gen), torch.randint(0, 9, (n,), generator=gen).float() * 2.0 ** -149, torch.randn(n, generator=gen) * 1e-30,
            torch.randint(-3, 1, (n,), generator=gen).float() * 2.0 ** -140]
    rows[0][: n // 3] = float("-inf")
    u = torch.tensor([0.9]).cuda()
    k = torch.ones(1, dtype=torch.int32).cuda()
    for row in rows:
        for temperature in (1.0, 0.3, 2.0, 4.0, 1e10, 1e30, 3e38, float("inf")):
            want = first_of_the_order(row, temperature)
            t = torch.tensor([temperature]).cuda()
            for p in (None, torch.tensor([0.5]).cuda()):
                token, logprob = rls.sample(row[None].cuda(), u, temperature=t, top_k=k, top_p=p)
                assert token.item() == want and logprob.item() == 0.0, (temperature, p)
    # a greedy row: the order of temperature 1
    for temperature in (0.0, -1.0, float("nan")):
        token, logprob = rls.sample(rows[1][None].cuda(), u, temperature=torch.tensor([temperature]).cuda())
        assert token.item() == first_of_the_order(rows[1], 1.0) and logprob.item() == 0.0
