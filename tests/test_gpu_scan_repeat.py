"""A linear scan gives the same bits whatever its tiles find when they look back: a composition, a state, or nothing in time.

With a wait limit of 0 every tile whose first look finds something missing goes through the tiles before it by itself, and from call to call
tiles find states at different distances.  Gates next to 1, so that an early step's rounding is still there at the end."""
import ctypes

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


def make(B, T, C, dtype, gate, resets):
    gen = torch.Generator(device="cuda").manual_seed(T + C)
    draw = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")      # noqa: E731
    a = torch.sigmoid(draw(B, T, C) + 8.0).to(gate)
    reset = (torch.rand(B, T, generator=gen, device="cuda") < 1.0 / 700).to(torch.uint8) if resets else None
    return a, draw(B, T, C).to(dtype), draw(B, T, C).to(dtype), draw(B, C), reset


CASES = [(1, 65521, 40, torch.float32, torch.float32, False), (1, 20000, 1024, torch.bfloat16, torch.float32, False), (3, 9000, 130, torch.float16, torch.float16, True),
         (2, 5000, 70, torch.float32, torch.float32, True), (1, 300007, 3, torch.float32, torch.float32, False), (1, 100000, 4, torch.bfloat16, torch.bfloat16, True),
         (3, 1000003, 1, torch.float32, torch.float32, False), (64, 65536, 1, torch.float32, torch.float32, True), (1, 5000011, 1, torch.bfloat16, torch.float32, False)]


@pytest.mark.parametrize("B,T,C,dtype,gate,resets", CASES)
def test_same_bits(rls, B, T, C, dtype, gate, resets):
    a, b, dh, h0, reset = make(B, T, C, dtype, gate, resets)
    limit = rls.lib().rls_scan_wait_limit
    limit.argtypes = [ctypes.c_int64]

    def both(reverse):
        h, last = rls.linear_scan(a, b, h0, reset, reverse)
        return h, last, *rls.linear_scan_backward(a, b, dh, h0, reset, h0, reverse)

    for reverse in (False, True):
        first = both(reverse)
        for ticks in (-1, 0, 0, 100, -1):
            assert limit(ticks) == 0
            try:
                again = both(reverse)
            finally:
                assert limit(-1) == 0
            assert all(torch.equal(x, y) for x, y in zip(first, again)), (reverse, ticks)
