"""Linear scans whose gates multiply up beyond the largest fp32 number while the states stay in range.

Powers of two make every step exact, so that a scan cut into tiles has to give what one step after the other gives, to the bit; other gates are
held to the error of fp32 arithmetic: a term that was carried over s steps is off by at most (s + 8) * 4 * 2^-24 of itself, as in any order of
evaluation that stays in range, and every state within the sum of that over its terms."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = [(2, 12, 128), (2, 40, 128), (1, 200, 128), (3, 300, 5), (1, 3000, 70), (2, 9000, 1), (1, 20000, 2), (1, 70000, 4), (2, 100, 1), (1, 33000, 1)]


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def limits(rls):
    """Both ways in which a tile learns what came before it."""
    limit = rls.lib().rls_scan_wait_limit
    limit.argtypes = [ctypes.c_int64]
    for ticks in (-1, 0):
        assert limit(ticks) == 0
        try:
            yield
        finally:
            assert limit(-1) == 0


@pytest.mark.parametrize("B,T,C", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_state_of_zero_under_large_gates(rls, B, T, C, dtype):
    """Gates of 4 and inputs of 0, until the last few steps: 0 until then."""
    a = torch.full((B, T, C), 4.0)
    b = torch.zeros(B, T, C)
    b[:, T - 6:] = 1.0
    want = torch.zeros(B, T, C)
    for t in range(T - 6, T):
        want[:, t] = 4.0 * want[:, t - 1] + 1.0                  # 1, 5, 21, 85, 341, 1365: 1365 takes 11 bits
    for _ in limits(rls):
        h, last = rls.linear_scan(a.cuda(), b.to(dtype).cuda())
        assert torch.equal(h.cpu(), want.to(dtype)) and torch.equal(last.cpu(), want[:, -1])
        h, last = rls.linear_scan(a.cuda().flip(1), b.to(dtype).cuda().flip(1), reverse=True)
        assert torch.equal(h.cpu().flip(1), want.to(dtype)) and torch.equal(last.cpu(), want[:, -1])
        # gradients of 0 until the first few steps, which come last
        da, db, dh0 = rls.linear_scan_backward(a.cuda(), torch.ones(B, T, C, dtype=dtype).cuda(), b.flip(1).to(dtype).cuda(), torch.ones(B, C).cuda())
        assert torch.equal(db.cpu().flip(1), want.to(dtype)) and torch.equal(da.cpu().flip(1), want) and torch.equal(dh0.cpu(), 4.0 * want[:, -1])


@pytest.mark.parametrize("B,T,C", SIZES)
@pytest.mark.parametrize("resets", [False, True])
def test_gates_that_undo_each_other(rls, B, T, C, resets):
    """2^100 twice, then 2^-100 twice: the state comes back, the product of the gates is infinite and then no number.  A reset begins anew."""
    pattern = torch.tensor([2.0 ** 100, 2.0 ** 100, 2.0 ** -100, 2.0 ** -100])
    a = pattern.repeat(T // 4 + 1)[:T][None, :, None].expand(B, T, C).contiguous()
    scale = (2.0 ** -torch.arange(1, C + 1).clamp(max=6).float())[None].expand(B, C)
    h0 = scale * 2.0 ** -110
    b = torch.zeros(B, T, C)
    reset = None
    h = h0.clone()
    if resets:
        reset = torch.zeros(B, T, dtype=torch.uint8)
        reset[:, 4 * (T // 8) - 1] = 1                           # (the last of a pattern)
        b[:, 4 * (T // 8) - 1] = scale * 2.0 ** -111
    want = torch.empty(B, T, C)
    for t in range(T):
        h = torch.where(reset[:, t, None] != 0, b[:, t], a[:, t] * h + b[:, t]) if resets else a[:, t] * h
        want[:, t] = h
    dev = lambda x: None if x is None else x.cuda()              # noqa: E731
    for _ in limits(rls):
        got, last = rls.linear_scan(a.cuda(), b.cuda(), h0.cuda(), dev(reset))
        assert torch.equal(got.cpu(), want) and torch.equal(last.cpu(), want[:, -1])
        # the same numbers, handed back from the last step: r_t = a_t r_{t+1}, g_t = r_{t+1}
        da, db, dh0 = rls.linear_scan_backward(a.flip(1).cuda(), torch.ones(B, T, C).cuda(), torch.zeros(B, T, C).cuda(), torch.ones(B, C).cuda(), None, h0.cuda())
        if not resets:
            want_db = torch.cat([h0[:, None], want[:, :-1]], 1).flip(1)
            assert torch.equal(db.cpu(), want_db) and torch.equal(da.cpu(), want_db) and torch.equal(dh0.cpu(), want[:, -1])


@pytest.mark.parametrize("B,T,C", SIZES)
def test_a_gate_of_zero_ends_a_run_of_large_ones(rls, B, T, C):
    """Large gates over a state of 0, a gate of 0, then ordinary gates and inputs."""
    gen = torch.Generator().manual_seed(T)
    a = torch.sigmoid(torch.randn(B, T, C, generator=gen) + 2.0)
    b = torch.randn(B, T, C, generator=gen)
    cut = T // 2
    a[:, :cut] = 1e30
    b[:, :cut] = 0.0
    a[:, cut] = 0.0
    x, y = a.double().numpy(), b.double().numpy()
    s, mags, weighted = np.zeros((B, C)), np.zeros((B, C)), np.zeros((B, C))
    want, slack = np.zeros((B, T, C)), np.zeros((B, T, C))
    for t in range(T):
        s = x[:, t] * s + y[:, t]
        mags = x[:, t] * mags + np.abs(y[:, t])
        weighted = x[:, t] * weighted + mags
        want[:, t], slack[:, t] = s, 4 * 2.0 ** -24 * (weighted + 8 * mags)
    for _ in limits(rls):
        h, last = rls.linear_scan(a.cuda(), b.cuda())
        assert (np.abs(h.double().cpu().numpy() - want) <= slack).all()
        assert (np.abs(last.double().cpu().numpy() - want[:, -1]) <= slack[:, -1]).all()


@pytest.mark.parametrize("B,T,C", SIZES)
def test_what_is_not_finite_stays_in_its_channel(rls, B, T, C):
    """One channel's inputs are not finite from some step on: it is not finite from there on, the others are as without it, and a reset ends it."""
    gen = torch.Generator().manual_seed(T + 1)
    a = torch.sigmoid(torch.randn(B, T, C, generator=gen) + 2.0)
    b = torch.randn(B, T, C, generator=gen)
    reset = torch.zeros(B, T, dtype=torch.uint8)
    reset[:, T - 3] = 1
    bad = b.clone()
    at = T // 3
    bad[:, at, C - 1] = float("inf")
    bad[:, at + 1, C - 1] = float("nan")
    clean, clean_last = rls.linear_scan(a.cuda(), b.cuda(), None, reset.cuda())
    for _ in limits(rls):
        h, last = rls.linear_scan(a.cuda(), bad.cuda(), None, reset.cuda())
        assert torch.equal(h[:, :, :C - 1], clean[:, :, :C - 1]) and torch.equal(h[:, T - 3:], clean[:, T - 3:]) and torch.equal(last, clean_last)
        assert torch.equal(h[:, :at], clean[:, :at]) and not torch.isfinite(h[:, at:T - 3, C - 1]).any()
