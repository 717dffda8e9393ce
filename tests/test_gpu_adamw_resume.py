"""An AdamW optimizer that takes over the moments of another one: the same steps from there on, and no moments in 8 bits without their scales."""
import pytest
import torch

pytestmark = pytest.mark.gpu

NAMES = ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def grads(seed):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(n, generator=gen).cuda() for n in (300, 5000)]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_resumed_run_goes_on(rls, bits):
    a = rls.AdamW(grads(0), state_bits=bits, seed=3)
    for k in range(3):
        a.step(grads(k + 1))
    held = {name: [t.clone() for t in getattr(a, name)] for name in NAMES if getattr(a, name) is not None}
    b = rls.AdamW([p.clone() for p in a.params], state_bits=bits, seed=3, step=3, **held)
    for opt in (a, b):
        opt.step(grads(9))
    assert all(torch.equal(x, y) for x, y in zip(a.params, b.params)) and all(torch.equal(x, y) for x, y in zip(a.exp_avg_sq, b.exp_avg_sq))


def test_codes_without_scales_and_scales_without_codes(rls):
    a = rls.AdamW(grads(0), state_bits=8)
    a.step(grads(1))
    for missing in NAMES:
        held = {name: [t.clone() for t in getattr(a, name)] for name in NAMES if name != missing}
        with pytest.raises(ValueError):
            rls.AdamW(grads(0), state_bits=8, step=1, **held)
        with pytest.raises(ValueError):
            rls.AdamW(grads(0), state_bits=8, step=1, **{missing: [t.clone() for t in getattr(a, missing)]})
