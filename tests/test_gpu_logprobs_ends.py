"""rls.token_logprobs and rls.distill_loss at the ends of their ranges: temperatures near 0 with factors above 1."""
import pytest
import torch

from tests.test_gpu_logprobs import TYPES, logits, rls                      # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [3, 12, 20, 100, 1000, 3000, 30000])
def test_gradients_at_tiny_temperatures(rls, n, kind):                          # noqa: F811
    """The largest logit is certain: its gradient is inv (factor - factor) = 0 however large inv is, and so is that of what has no probability.  Where another
    entry is the given one, inv times the factor lands there, and less it at the certain one: numbers, or infinities of the right sign, none of them NaN."""
    rows = 6
    x = logits(rows, n, kind, n)
    best = x.float().argmax(1)
    x.scatter_(1, best[:, None], 20.0)
    x[5] = -torch.inf                                                              # certain because nothing else is left
    x[5, best[5]] = 1.0
    t = torch.tensor([1e-40, 1e-38, 1e-37, 1e-30, 1e-3, 1e-40]).cuda()
    inv = (1.0 / t).clamp(max=2e38)
    tokens = best.to(torch.int32)
    other = ((best + 1) % n).to(torch.int32)
    r = rls.token_logprobs(x, tokens, temperature=t)
    assert not r.logprob.any() and not r.entropy.any()
    for factor in (10.0, -10.0, 0.25):
        by = torch.full((rows,), factor, device="cuda")
        for dentropy in (None, by):
            assert not rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, by, dentropy, temperature=t).any()
        got = rls.token_logprobs_backward(x, other, r.norm, r.entropy, by, by, temperature=t)
        want = torch.zeros_like(got, dtype=torch.float32)
        want.scatter_(1, best[:, None], -(inv * by)[:, None])
        want.scatter_(1, other.long()[:, None], (inv * by)[:, None])
        want[5, other[5]] = 0.0                                                    # (masked)
        assert torch.equal(got, want.to(got.dtype))

        # a teacher that is as certain: of the same entry, and of another
        for token, row in ((tokens, 0.0 * by), (other, by)):
            k = torch.stack([token, tokens, token], 1)
            scores = torch.tensor([3.0, -torch.inf, 3.0], device="cuda").expand(rows, 3).contiguous()
            loss, norm = rls.distill_loss(x, k, scores, temperature=t)
            got = rls.distill_loss_backward(x, k, scores, norm, by, temperature=t)
            want = torch.zeros_like(got, dtype=torch.float32)
            want.scatter_(1, best[:, None], (inv * row)[:, None])
            want.scatter_(1, token.long()[:, None], -(inv * row)[:, None])
            want[5, other[5]] = 0.0
            assert torch.equal(got, want.to(got.dtype)) and not loss.isnan().any()
