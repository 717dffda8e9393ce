"""The gated linear recurrence and its backward pass against their definition in 64 bits.

A state is a sum of products of gates and inputs.  With |a| <= 1 every term of fp32 arithmetic is off by at most a few rounding
errors per step it is carried over, whatever the order of the steps is cut into: |error| <= 4 * 2^-24 * sum over the terms of
(steps carried + 8) * |term|, which the reference computes beside the states (the recurrence on absolute values, and once more on those).
What is stored in fewer bits takes one rounding to its type on top, 2^-8 (bf16) or 2^-11 (fp16, and 2^-25 absolute where it is subnormal) of the value.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().double().cpu().numpy()


def recurrence(a, b, s):
    h = np.empty_like(b)
    for t in range(b.shape[1]):
        s = a[:, t] * s + b[:, t]
        h[:, t] = s
    return h, s


def bounded(a, b, s):
    """States, the last one, and for every state what its fp32 error may be."""
    h, last = recurrence(a, b, s)
    mags, _ = recurrence(np.abs(a), np.abs(b), np.abs(s))
    weighted, _ = recurrence(np.abs(a), mags, np.abs(s))
    return h, last, 4 * 2.0 ** -24 * (weighted + 8 * mags)


def effective(a, reset, reverse):
    a = a.copy()
    if reset is not None:
        a[reset != 0] = 0.0
    return a[:, ::-1] if reverse else a


def near(got, want, slack, dtype, name):
    got = f64(got)
    allowed = slack + HALF_STEP[dtype] * (np.abs(want) + slack) + (2.0 ** -24 if dtype == torch.float16 else 2.0 ** -140)
    bad = ~(np.abs(got - want) <= allowed)
    assert not bad.any(), (name, np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], allowed[bad][:5])


def make(B, T, C, dtype, gate, seed, with_h0=True, with_reset=False, centre=2.0):
    gen = torch.Generator().manual_seed(seed)
    a = torch.sigmoid(torch.randn(B, T, C, generator=gen) + centre).to(gate)
    if T > 2:
        a[:, T // 2, ::3] *= -1
    b = torch.randn(B, T, C, generator=gen).to(dtype)
    h0 = torch.randn(B, C, generator=gen) if with_h0 else None
    reset = (torch.rand(B, T, generator=gen) < 0.1).to(torch.uint8) if with_reset else None
    return a, b, h0, reset


def dev(t):
    return None if t is None else t.cuda()


def np_of(t):
    return None if t is None else t.numpy()


def check_forward(rls, a, b, h0, reset, reverse, a_dev=None, b_dev=None, **calls):
    h, last = rls.linear_scan(dev(a) if a_dev is None else a_dev, dev(b) if b_dev is None else b_dev, dev(h0), dev(reset), reverse, **calls)
    s = np.zeros((a.shape[0], a.shape[2])) if h0 is None else f64(h0)
    ae, be = effective(f64(a), np_of(reset), reverse), f64(b)
    want, want_last, slack = bounded(ae, be[:, ::-1] if reverse else be, s)
    turn = (lambda x: x[:, ::-1]) if reverse else (lambda x: x)
    near(h, turn(want), turn(slack), b.dtype, "h")
    near(last, want_last, slack[:, -1], torch.float32, "last")
    return h, last


def check_backward(rls, a, h, dh, h0, reset, dlast, reverse, a_dev=None, dh_dev=None):
    da, db, dh0 = rls.linear_scan_backward(dev(a) if a_dev is None else a_dev, dev(h), dev(dh) if dh_dev is None else dh_dev, dev(h0), dev(reset),
                                           dev(dlast), reverse)
    B, T, C = a.shape
    turn = (lambda x: x[:, ::-1]) if reverse else (lambda x: x)
    ae, he, dhe = effective(f64(a), np_of(reset), reverse), turn(f64(h)), turn(f64(dh)).copy()
    s0 = np.zeros((B, C)) if h0 is None else f64(h0)
    dhe[:, -1] += 0.0 if dlast is None else f64(dlast)
    back = np.concatenate([ae[:, 1:], np.zeros((B, 1, C))], 1)
    g, _, slack = bounded(back[:, ::-1], dhe[:, ::-1], np.zeros((B, C)))
    g, slack = g[:, ::-1], slack[:, ::-1]
    before = np.concatenate([s0[:, None], he[:, :-1]], 1)
    want_da = g * before
    if reset is not None:
        want_da[turn(np_of(reset)) != 0] = 0.0
    near(db, turn(g), turn(slack), dh.dtype, "db")
    near(da, turn(want_da), turn(slack * np.abs(before) + 2.0 ** -24 * np.abs(want_da)), a.dtype, "da")
    near(dh0, ae[:, 0] * g[:, 0], np.abs(ae[:, 0]) * slack[:, 0], torch.float32, "dh0")
    return da, db, dh0


SIZES = [(1, 1, 1), (3, 1, 5), (64, 1, 130), (2, 2, 64), (1, 7, 3), (3, 63, 65), (2, 64, 128), (1, 129, 257), (5, 300, 33), (1, 1025, 48), (2, 4099, 19),
         (1, 20001, 8), (300, 40, 70), (2, 513, 1024), (130, 24, 1030), (70000, 60, 1)]


@pytest.mark.parametrize("B,T,C", SIZES)
@pytest.mark.parametrize("dtype,gate", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f16", "f32")])
def test_both_directions_against_64_bits(rls, B, T, C, dtype, gate):
    for reverse in (False, True):
        seed = B * T + C + reverse
        a, b, h0, reset = make(B, T, C, TYPES[dtype], TYPES[gate], seed, with_h0=seed % 2 == 0, with_reset=seed % 3 == 0)
        h, _ = check_forward(rls, a, b, h0, reset, reverse)
        gen = torch.Generator().manual_seed(seed + 1)
        dh = torch.randn(B, T, C, generator=gen).to(TYPES[dtype])
        check_backward(rls, a, h.cpu(), dh, h0, reset, torch.randn(B, C, generator=gen) if seed % 2 else None, reverse)


@pytest.mark.parametrize("B,T", [(1, 1), (1, 5), (3, 64), (2, 1000), (1, 1024), (1, 8193), (4, 30001), (1, 300007), (70, 999)])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("resets", [False, True])
def test_returns(rls, B, T, reverse, resets):
    """One channel: discounted sums over a trajectory, cut into episodes."""
    gen = torch.Generator().manual_seed(B + T)
    a = torch.full((B, T, 1), 0.9 * 0.99)
    b = torch.randn(B, T, 1, generator=gen)
    reset = (torch.rand(B, T, generator=gen) < 0.01).to(torch.uint8) if resets else None
    h0 = torch.randn(B, 1, generator=gen)
    h, _ = check_forward(rls, a, b, h0, reset, reverse)
    check_backward(rls, a, h.cpu(), torch.randn(B, T, 1, generator=gen), h0, reset, torch.randn(B, 1, generator=gen), reverse)


@pytest.mark.parametrize("B,T,C", [(1, 40000, 16), (1, 9000, 130), (2, 70001, 1)])
def test_long_memory(rls, B, T, C):
    """Gates next to 1: a state remembers thousands of steps, across every cut of the time axis."""
    a, b, h0, _ = make(B, T, C, torch.float32, torch.float32, T, centre=8.0)
    h, _ = check_forward(rls, a, b, h0, None, False)
    check_backward(rls, a, h.cpu(), torch.randn(B, T, C, generator=torch.Generator().manual_seed(1)), h0, None, None, False)


@pytest.mark.parametrize("B,T,C", [(1, 5000, 64), (3, 2048, 1), (2, 700, 96)])
def test_gates_of_one_and_zero(rls, B, T, C):
    """a = 1 counts exactly (whole numbers below 2^24), a = 0 copies the input."""
    ones = torch.ones(B, T, C).cuda()
    h, last = rls.linear_scan(ones, ones)
    want = torch.arange(1, T + 1, device="cuda").float()[None, :, None].expand(B, T, C)
    assert torch.equal(h, want) and (last == T).all()
    b = torch.randn(B, T, C).cuda()
    h, last = rls.linear_scan(torch.zeros(B, T, C).cuda(), b)
    assert torch.equal(h, b) and torch.equal(last, b[:, -1])


def test_a_reset_drops_what_is_not_finite(rls):
    """Infinities and NaN before a reset stay before it, in both passes; a gate that is not finite has no part in its step."""
    for B, T, C in ((1, 200, 3), (2, 3000, 1), (1, 5000, 70)):
        for reverse in (False, True):
            a, b, h0, _ = make(B, T, C, torch.float32, torch.float32, 5)
            cut = T // 2
            reset = torch.zeros(B, T, dtype=torch.uint8)
            reset[:, cut] = 1
            a[:, cut] = float("nan")
            early = slice(cut + 1, T) if reverse else slice(0, cut)
            late = slice(0, cut + 1) if reverse else slice(cut, T)
            b[:, early] = float("inf")
            h0[:] = float("nan")
            h, last = rls.linear_scan(dev(a), dev(b), dev(h0), dev(reset), reverse)
            assert torch.isfinite(h[:, late]).all() and torch.isfinite(last).all() and not torch.isfinite(h[:, early]).any()
            dh = torch.randn(B, T, C)
            dh[:, late] = float("nan")
            h = torch.randn(B, T, C)
            da, db, dh0 = rls.linear_scan_backward(dev(a), dev(h), dev(dh), torch.zeros(B, C).cuda(), dev(reset), None, reverse)
            assert torch.isfinite(db[:, early]).all() and torch.isfinite(da[:, early]).all() and torch.isfinite(dh0).all()
            assert (da[:, cut] == 0).all() and torch.isnan(db[:, late]).all()


def test_no_steps(rls):
    h0 = torch.randn(3, 5).cuda()
    a = torch.empty(3, 0, 5).cuda()
    h, last = rls.linear_scan(a, a, h0)
    assert h.shape == (3, 0, 5) and torch.equal(last, h0)
    h, last = rls.linear_scan(a, a)
    assert (last == 0).all()
    da, db, dh0 = rls.linear_scan_backward(a, a, a, h0, dh_last=h0)
    assert da.shape == db.shape == (3, 0, 5) and torch.equal(dh0, h0)


@pytest.mark.parametrize("B,T,C", [(2, 300, 65), (1, 6000, 40), (3, 500, 1)])
def test_strides_and_broadcasts(rls, B, T, C):
    """Views of larger arrays, time before the sequences, odd starts, inputs that repeat themselves."""
    gen = torch.Generator().manual_seed(T)
    a, b, h0, reset = make(B, T, C, torch.bfloat16, torch.float32, 3, with_reset=True)
    wide = torch.full((B, T, 2 * C + 3), float("nan"), dtype=torch.bfloat16).cuda()
    wide[:, :, 1:1 + C] = b.cuda()
    turned = torch.empty(T, B, C).cuda().copy_(a.cuda().transpose(0, 1)).transpose(0, 1)
    out = torch.full((T, B, C + 5), 7.0, dtype=torch.bfloat16).cuda()
    check_forward(rls, a, b, h0, reset, False, a_dev=turned, b_dev=wide[:, :, 1:1 + C], out=out[:, :, 2:2 + C].transpose(0, 1))
    assert (out[:, :, :2] == 7).all() and (out[:, :, 2 + C:] == 7).all()
    gate = torch.sigmoid(torch.randn(C, generator=gen))
    check_forward(rls, gate.expand(B, T, C), b, h0, None, True, a_dev=gate.cuda().expand(B, T, C))
    per_step = torch.sigmoid(torch.randn(1, T, C, generator=gen))
    h, _ = check_forward(rls, per_step.expand(B, T, C), b, h0, None, False, a_dev=per_step.cuda().expand(B, T, C))
    dh = torch.randn(B, T, C, generator=gen).to(torch.bfloat16)
    wide[:, :, C + 2:2 * C + 2] = dh.cuda()
    check_backward(rls, per_step.expand(B, T, C), h.cpu(), dh, h0, reset, None, False, a_dev=per_step.cuda().expand(B, T, C),
                   dh_dev=wide[:, :, C + 2:2 * C + 2])


@pytest.mark.parametrize("B,T,C", [(64, 1, 100), (2, 5000, 33), (1, 20000, 1)])
def test_state_updated_in_place(rls, B, T, C):
    """h_last in h0's memory, dh0 in dh_last's: same results as apart, one token or many."""
    a, b, h0, reset = make(B, T, C, torch.float32, torch.float32, 11)
    want_h, want = rls.linear_scan(dev(a), dev(b), dev(h0))
    state = h0.cuda()
    h, last = rls.linear_scan(dev(a), dev(b), state, last=state)
    assert last is state and torch.equal(state, want) and torch.equal(h, want_h)
    # token by token, the state handed on
    if T > 1 and T <= 5000:
        state = h0.cuda()
        for t in range(5):
            rls.linear_scan(dev(a[:, t:t + 1]), dev(b[:, t:t + 1]), state, last=state)
        h5, last5 = rls.linear_scan(dev(a[:, :5].contiguous()), dev(b[:, :5].contiguous()), dev(h0))
        assert torch.equal(state, last5)


@pytest.mark.parametrize("B,T,C", [(1, 37, 3), (2, 600, 2), (1, 3000, 1)])
def test_gradients_against_differences(rls, B, T, C):
    """L = <h, r> + <last, r_last> is linear in each single gate, input and state: its difference over a whole step is the derivative, up to the fp32 errors of
    the states that both sides are summed from (in 64 bits), and the gradient's own."""
    gen = torch.Generator().manual_seed(T)
    a, b, h0, reset = make(B, T, C, torch.float32, torch.float32, 21, with_reset=True)
    r, r_last = torch.randn(B, T, C, generator=gen), torch.randn(B, C, generator=gen)
    h, _ = rls.linear_scan(dev(a), dev(b), dev(h0), dev(reset))
    da, db, dh0 = rls.linear_scan_backward(dev(a), h, dev(r), dev(h0), dev(reset), dev(r_last))

    def loss(a, b, h0):
        h, last = rls.linear_scan(dev(a), dev(b), dev(h0), dev(reset))
        _, _, slack = bounded(effective(f64(a), np_of(reset), False), f64(b), f64(h0))
        error = (slack * r.abs().numpy()).sum() + (slack[:, -1] * r_last.abs().numpy()).sum()
        return float((h.double().cpu() * r).sum() + (last.double().cpu() * r_last).sum()), error

    for which, grad in ((0, da), (1, db), (2, dh0)):
        for _ in range(6):
            at = tuple(int(torch.randint(0, n, (1,), generator=gen)) for n in (a, b, h0)[which].shape)
            values, errors = [], 0.0
            for side in (0.5, -0.5):
                x = [a.clone(), b.clone(), h0.clone()]
                x[which][at] += side
                value, error = loss(*x)
                values.append(value)
                errors += error
            slope = values[0] - values[1]
            assert abs(slope - float(grad[at])) <= errors + 2.0 ** -18 * abs(slope), (which, at)


@pytest.mark.parametrize("B,T,C,dtype", [(1, 3000, 70, "bf16"), (2, 1500, 3, "f32"), (2, 20000, 1, "f32"), (3, 4100, 200, "f32")])
def test_tiles_that_do_not_wait(rls, B, T, C, dtype):
    """Tiles that give up at once on what is not there yet go through the steps before them by themselves."""
    import ctypes
    a, b, h0, reset = make(B, T, C, TYPES[dtype], torch.float32, 4, with_reset=True)
    limit = rls.lib().rls_scan_wait_limit
    limit.argtypes = [ctypes.c_int64]
    assert limit(0) == 0
    try:
        for reverse in (False, True):
            h, _ = check_forward(rls, a, b, h0, reset, reverse)
            check_backward(rls, a, h.cpu(), torch.randn(B, T, C, generator=torch.Generator().manual_seed(1)).to(TYPES[dtype]), h0, reset, h0, reverse)
    finally:
        assert limit(-1) == 0


def test_in_a_graph(rls):
    for B, T, C in ((64, 1, 96), (1, 20000, 24), (2, 30000, 1)):
        a, b = torch.empty(B, T, C).cuda(), torch.empty(B, T, C).cuda()
        ws = torch.empty(rls.linear_scan_workspace_bytes(B, T, C) + 256, dtype=torch.uint8).cuda()
        out, last = torch.empty(B, T, C).cuda(), torch.empty(B, C).cuda()
        a.uniform_(0, 1), b.normal_()
        rls.linear_scan(a, b, workspace=ws, out=out, last=last)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            rls.linear_scan(a, b, workspace=ws, out=out, last=last)
        for _ in range(4):
            a.uniform_(0, 1), b.normal_()
            want, want_last = rls.linear_scan(a, b)
            out.zero_(), last.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want) and torch.equal(last, want_last)


def test_same_result_every_time(rls):
    for B, T, C in ((1, 65521, 40), (3, 100000, 1)):
        a, b, h0, _ = make(B, T, C, torch.float32, torch.float32, 2)
        first = rls.linear_scan(dev(a), dev(b), dev(h0))
        for _ in range(3):
            again = rls.linear_scan(dev(a), dev(b), dev(h0))
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("T,C", [(12, 70), (70, 70), (70, 2)])
def test_offsets_beyond_32_bits(rls, T, C):
    """Steps 2^26 elements apart: the last ones lie past 2^32 bytes."""
    a, b, h0, _ = make(1, T, C, torch.bfloat16, torch.float32, T)
    apart = (1 << 26) if T > 60 else (1 << 28)
    whole = torch.empty(T * apart, dtype=torch.bfloat16, device="cuda")
    far = whole.view(1, T, apart)[:, :, apart - C:]
    far.copy_(b)
    h, _ = check_forward(rls, a, b, h0, None, False, b_dev=far)
    dh = torch.randn(1, T, C, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    far.copy_(dh)
    check_backward(rls, a, h.cpu(), dh, h0, None, None, False, dh_dev=far)
    out = far                                            # written through as well
    h2, _ = rls.linear_scan(dev(a), dev(b), dev(h0), out=out)
    assert torch.equal(h2, h)


def test_nothing_around_the_outputs_is_written(rls):
    """Odd sizes inside larger arrays, both passes: the border keeps what it held."""
    for B, T, C in ((2, 300, 67), (1, 1000, 3), (2, 5000, 1), (3, 20, 130)):
        a, b, h0, _ = make(B, T, C, torch.bfloat16, torch.bfloat16, 8)
        border = torch.full((B + 2, T + 2, C + 4), 3.0, dtype=torch.bfloat16).cuda()
        out = border[1:1 + B, 1:1 + T, 2:2 + C]
        want, _ = rls.linear_scan(dev(a), dev(b), dev(h0))
        rls.linear_scan(dev(a), dev(b), dev(h0), out=out)
        assert torch.equal(out, want)
        border[1:1 + B, 1:1 + T, 2:2 + C] = 3.0
        assert (border == 3).all()
