"""The factor of the gradients in an AdamW step, from the smallest to the largest (clipping after a jump, loss scaling), against the definition in 64 bits.

The bounds are those of a step without a factor: m and v take three roundings each, 2^-22 of the sum of their terms' magnitudes with one to spare; the root
and the quotient of the update, from m and v off by that much, at most 2^-20 of it; the weight three roundings of its own.  Gradients that the factor
brings below the smallest normal number lose bits there: 2^-149 a gradient."""
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


@pytest.mark.parametrize("scale", [1.0, 0.37, -3.0, 1e-3, 2.0 ** 16, 3e-18, 1e-22, 7e-30, 1e-37, 1e-42, 5e18, 1e25, 3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_any_factor(rls, scale, dtype):
    gen = torch.Generator().manual_seed(7)
    n, lr, b1, b2, eps, wd = 3000, 1e-2, 0.9, 0.99, 1e-8, 0.1
    factor = torch.tensor([scale], dtype=torch.float32)
    exact = float(factor.double())
    size = min(max(1.0 / abs(exact), 1e-37), 1e37)                     # gradients that the factor brings to about 1, as far as there are any
    grad = (torch.randn(n, generator=gen).double() * size).to(dtype)
    grad = torch.where(grad.abs().double() < 2.0 ** -126, torch.zeros_like(grad), grad)
    p, m, v = torch.randn(n, generator=gen), torch.randn(n, generator=gen) * 0.1, torch.rand(n, generator=gen) * 0.1
    dev = [x.clone().cuda() for x in (p, m, v)]
    opt = rls.AdamW([dev[0].to(dtype)], master=[dev[0]] if dtype != torch.float32 else None, exp_avg=[dev[1]], exp_avg_sq=[dev[2]], step=4)
    opt.step([grad.cuda()], lr=lr, betas=(b1, b2), eps=eps, weight_decay=wd, grad_scale=factor.cuda())
    g = grad.double().numpy() * exact
    p0, m0, v0 = (x.double().numpy() for x in (p, m, v))
    lost = 2.0 ** -149
    m1, v1 = b1 * m0 + (1 - b1) * g, b2 * v0 + (1 - b2) * g * g
    mags = b1 * np.abs(m0) + (1 - b1) * np.abs(g)
    root = np.sqrt(v1 / (1 - b2 ** 5)) + eps
    update, spread = lr / (1 - b1 ** 5) * m1 / root, lr / (1 - b1 ** 5) * mags / root
    got_m, got_v = opt.exp_avg[0].double().cpu().numpy(), opt.exp_avg_sq[0].double().cpu().numpy()
    assert (np.abs(got_m - m1) <= 2.0 ** -22 * mags + 2 * lost).all()
    assert (np.abs(got_v - v1) <= 2.0 ** -22 * v1 + 2 * lost * (1 + np.abs(g))).all()
    weight = (opt.master[0] if dtype != torch.float32 else opt.params[0]).double().cpu().numpy()
    want = p0 * (1 - lr * wd) - update
    assert (np.abs(weight - want) <= 3 * 2.0 ** -24 * np.abs(p0) + 2.0 ** -20 * spread).all()


def test_factors_that_are_no_numbers(rls):
    """They reach every parameter, as the formula has it; a factor of 0 is a gradient of 0."""
    for value in (float("inf"), float("-inf"), float("nan"), 0.0):
        for bits in (32, 8):
            opt = rls.AdamW([torch.ones(700).cuda()], state_bits=bits)
            opt.step([torch.full((700,), 0.5).cuda()], weight_decay=0.0, grad_scale=torch.tensor([value]).cuda())
            if value == 0.0:
                assert (opt.params[0] == 1.0).all()
            else:
                assert torch.isnan(opt.params[0]).all()
