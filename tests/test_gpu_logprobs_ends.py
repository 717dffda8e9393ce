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


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [1, 3, 16, 40, 300, 1025, 20000, 70000])
def test_beside_an_infinite_logit(rls, n, kind):                                 # noqa: F811
    """+infinity counts as the largest fp32 number: it is certain, and any other entry has that number less of log p; with half the temperature, more than there is."""
    largest = torch.finfo(torch.float32).max
    x = logits(3, n, kind, n)
    x[:, n // 3] = torch.inf
    tokens = torch.tensor([n // 2, n // 3, n // 2], dtype=torch.int32, device="cuda")
    t = torch.tensor([1.0, 1.0, 0.5], device="cuda")
    r = rls.token_logprobs(x, tokens, temperature=t, top=1)
    same = n // 2 == n // 3
    assert r.logprob.tolist() == ([0.0, 0.0, 0.0] if same else [-largest, 0.0, -torch.inf])
    assert bool((r.top_token[:, 0] == n // 3).all()) and not r.top_logprob.any() and not r.entropy.any() and bool((r.norm[:, 0] == largest).all())
    by = torch.full((3,), 0.75, device="cuda")
    got, want = rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, by, by, temperature=t), torch.zeros(3, n, device="cuda")
    if not same:
        for row in (0, 2):
            want[row, n // 3], want[row, n // 2] = -0.75 / t[row], 0.75 / t[row]
    assert torch.equal(got, want.to(got.dtype))


def test_whole_rows_past_32_bits(rls):                                           # noqa: F811
    """Rows that begin beyond 2^31 entries, all of their gradients, and of the teacher's: the same bits as those rows by themselves."""
    rows, n, k = 133, 1 << 24, 4
    x = torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda")
    x[-2:] = logits(2, n, "bf16", 1)
    tokens = torch.full((rows,), n - 1, dtype=torch.int32, device="cuda")
    tokens[-2] = n // 3
    parts = [slice(0, 1), slice(rows - 5, rows - 3), slice(rows - 2, rows)]       # (the second is at 2^31)
    assert (rows - 5) * n == 1 << 31
    few = [x[p].clone() for p in parts]
    r = rls.token_logprobs(x, tokens)
    by = torch.linspace(-1.0, 1.0, rows, device="cuda")
    teacher = (n - 1 - 7 * torch.arange(k, device="cuda")).expand(rows, k).to(torch.int32).contiguous()
    scores = torch.arange(k, dtype=torch.float32, device="cuda").expand(rows, k).contiguous()
    loss, norm = rls.distill_loss(x, teacher, scores)
    for p, y in zip(parts, few):
        one = rls.token_logprobs(y, tokens[p].clone())
        l1, n1 = rls.distill_loss(y, teacher[p].clone(), scores[p].clone())
        # sums in other parts of the rows: 64 roundings and those of 2^24 / 256 additions in a row
        tol = 2.0 ** -24 * ((1 << 16) + 64)
        for a, b in ((r.logprob[p], one.logprob), (r.entropy[p], one.entropy), (r.norm[p], one.norm), (loss[p], l1), (norm[p], n1)):
            assert float((a - b).abs().max()) <= tol * (1 + float(b.abs().max()))
    want = [(rls.token_logprobs_backward(y, tokens[p].clone(), r.norm[p].clone(), r.entropy[p].clone(), by[p].clone(), by[p].clone()),
             rls.distill_loss_backward(y, teacher[p].clone(), scores[p].clone(), norm[p].clone(), by[p].clone())) for p, y in zip(parts, few)]
    out = torch.empty_like(x)
    rls.distill_loss_backward(x, teacher, scores, norm, by, out=out)
    assert all(torch.equal(out[p], w[1]) for p, w in zip(parts, want))
    rls.token_logprobs_backward(x, tokens, r.norm, r.entropy, by, by, out=x)
    assert all(torch.equal(x[p], w[0]) for p, w in zip(parts, want))
    assert all(bool(w[0].any()) and bool(w[1].any()) for w in want)
