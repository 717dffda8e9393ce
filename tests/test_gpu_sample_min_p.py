"""min-p from 1 on: entries whose exponential is 1 stay, all of them, at every length of rows; what lies below goes."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("n", [5, 16, 20, 50, 100, 900, 12000, 30000, 140001])
@pytest.mark.parametrize("min_p", [1.0, 1.5, 3.0, float("inf")])
def test_ties_and_near_ties(rls, n, min_p):
    """A fifth of the entries at the largest value, a fifth 2^-40 below it (its exponential is 1 in fp32), the others 2^-10 below and further down."""
    rows = 8
    logits = torch.zeros(rows, n)
    logits[:, 1::5] = -(2.0 ** -40)
    logits[:, 2::5] = -(2.0 ** -10)
    logits[:, 3::5] = -3.0
    logits[:, 4::5] = float("-inf")
    kept = np.flatnonzero((np.arange(n) % 5) < 2)
    u = (torch.arange(rows).float() + 0.5) / rows
    m = torch.full((rows,), min_p)
    for top_p in (None, torch.full((rows,), 0.999).cuda()):
        token, logprob = rls.sample(logits.cuda(), u.cuda(), min_p=m.cuda(), top_p=top_p)
        for r in range(rows):
            if top_p is None:
                # equal weights: the floor(u * kept)-th, whole numbers throughout
                assert token[r].item() == kept[int(np.float64(u[r].item()) * len(kept))], r
            assert token[r].item() in kept and abs(logprob[r].item() + np.log(len(kept))) <= 2.0 ** -17 * (1 + np.log(len(kept)))
