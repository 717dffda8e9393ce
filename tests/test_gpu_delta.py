"""rls.gated_delta against the recurrence step by step in 64 bits, and its gradients against that loop's.

Keys have length 1 and beta is at most 1, so a step never lengthens an error: the ones of T steps, each a sum over the key dimensions, in chunks over 64 steps too,
add up like independent ones.  Tolerances are 8 times 2^-24 sqrt((T + 64) (key_dim + 64)) of the largest value, twice as much for gradients (a product
of two such sums each), and half a step of the result's type."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def loop(q, k, v, g, beta, state, reset, scale):
    """In 64 bits, step by step."""
    q, k, v, g, beta = (x.double() for x in (q, k, v, g, beta))
    group = v.shape[2] // q.shape[2]
    q, k = q.repeat_interleave(group, 2), k.repeat_interleave(group, 2)
    B, T, H, V = v.shape
    s = torch.zeros(B, H, q.shape[3], V, dtype=torch.float64, device=v.device) if state is None else state.double()
    out = []
    for t in range(T):
        carried = torch.exp(g[:, t])[:, :, None, None] * s
        if reset is not None:
            carried = torch.where(reset[:, t, None, None, None] != 0, 0.0, carried)
        y = v[:, t] - (carried * k[:, t, :, :, None]).sum(2)
        s = carried + k[:, t, :, :, None] * (beta[:, t, :, None] * y)[:, :, None]
        out.append(scale * (s * q[:, t, :, :, None]).sum(2))
    return (torch.stack(out, 1) if out else v.new_zeros(B, 0, H, V)), s


def inputs(B, T, H, HK, K, V, kind, seed, reset=False, state=True):
    gen = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(*shape, generator=gen)             # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)                    # noqa: E731
    d = {"q": unit(draw(B, T, HK, K)), "k": unit(draw(B, T, HK, K)), "v": draw(B, T, H, V)}
    d = {n: x.to(TYPES[kind]).cuda() for n, x in d.items()}
    d["g"] = -torch.nn.functional.softplus(2 * draw(B, T, H) - 2).cuda()
    d["beta"] = torch.sigmoid(draw(B, T, H)).cuda()
    d["state"] = draw(B, H, K, V).cuda() if state else None
    d["reset"] = (torch.rand(B, T, generator=gen) < 0.03).to(torch.uint8).cuda() if reset else None
    return d


def close(got, want, T, K, twice, what, terms=0.0):
    """terms: the largest of what cancels in `want`."""
    if want.numel() == 0:
        assert got.shape == want.shape
        return
    kind = torch.finfo(got.dtype)
    g, w = got.double(), want.double()
    assert g.shape == w.shape and bool(g.isfinite().all()), what
    tol = twice * 8 * UNIT * ((T + 64) * (K + 64)) ** 0.5 * max(float(w.abs().max()), float(terms)) + (w.abs() * kind.eps / 2 * 1.001 + kind.smallest_normal * kind.eps if got.dtype != torch.float32 else 0)
    off = (g - w).abs()
    assert bool((off <= tol).all()), (what, float(off.max()), float(w.abs().max()))


SHAPES = [(1, 1, 1, 1, 1, 1), (2, 1, 4, 2, 128, 128), (3, 5, 3, 1, 17, 130), (2, 8, 2, 2, 33, 5), (1, 9, 2, 1, 64, 64), (2, 37, 4, 4, 64, 64), (1, 63, 1, 1, 16, 16),
          (1, 64, 2, 1, 32, 100), (2, 65, 2, 2, 128, 128), (1, 128, 1, 1, 100, 33), (3, 130, 6, 2, 40, 72), (2, 300, 3, 3, 65, 200), (1, 700, 4, 1, 128, 64), (9, 70, 1, 1, 20, 512), (64, 12, 4, 2, 16, 24), (65, 16, 4, 4, 24, 70)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(rls, shape, kind):
    for reset, state in ((False, True), (True, True), (True, False)):
        d = inputs(*shape, kind, sum(shape), reset, state)
        o, last = rls.gated_delta(**d)
        want, end = loop(*d.values(), shape[4] ** -0.5)
        close(o, want, shape[1], shape[4], 1, "o")
        close(last, end, shape[1], shape[4], 1, "last")


def gradients(d, do, dlast, scale):
    leaves = {n: x.double().requires_grad_() for n, x in d.items() if n != "reset" and x is not None}
    o, last = loop(**{**d, **leaves}, scale=scale)
    value = (o * do.double()).sum() + (0 if dlast is None else (last * dlast.double()).sum())
    return dict(zip(leaves, torch.autograd.grad(value, list(leaves.values()))))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(rls, shape, kind):
    B, T, H, HK, K, V = shape
    gen = torch.Generator().manual_seed(T)
    do, dlast = torch.randn(B, T, H, V, generator=gen).to(TYPES[kind]).cuda(), torch.randn(B, H, K, V, generator=gen).cuda()
    for reset, state in ((False, True), (True, False)):
        d = inputs(*shape, kind, sum(shape), reset, state)
        got = dict(zip(("q", "k", "v", "g", "beta", "state"), rls.gated_delta_backward(**{n: d[n] for n in ("q", "k", "v", "g", "beta")}, do=do, state=d["state"],
                                                                                       reset=d["reset"], dlast=dlast if state else None, scale=0.3)))
        want = gradients(d, do, dlast if state else None, 0.3)
        if reset:
            want["g"] = want["g"].masked_fill(d["reset"][:, :, None] != 0, 0.0)
        # dg_t is the sum over the steps from t on of what their decays take part in, less beta dbeta: a rounding of that is 2^-24 |beta dbeta|, also where
        # all of it cancels (a first step without a state)
        terms = (d["beta"] * want["beta"]).abs().max()
        for n, w in want.items():
            close(got[n], w, T, K, 2, n, terms if n == "g" else 0.0)


@pytest.fixture
def short_segments(rls):
    """Chunks of a few launches each, as with long sequences of many heads."""
    set_bytes = rls.lib().rls_delta_segment_bytes
    set_bytes.argtypes = [ctypes.c_int64]
    yield lambda n: set_bytes(n)
    set_bytes(-1)


@pytest.mark.parametrize("chunks", [1, 2, 3])
def test_segments(rls, short_segments, chunks):
    B, T, H, HK, K, V = shape = (2, 450, 2, 1, 64, 64)
    d = inputs(*shape, "f32", 3, True)
    do, dlast = torch.randn(B, T, H, V).cuda(), torch.randn(B, H, K, V).cuda()
    args = [d[n] for n in ("q", "k", "v", "g", "beta")]
    whole = rls.gated_delta(**d), rls.gated_delta_backward(*args, do, d["state"], d["reset"], dlast)
    for per_chunk, backward in ((4 * (2 * 4096 + 4096 + 4096), False), (4 * (2 * 4096 + 2 * 8192 + 4096 + 2 * 4096), True)):
        short_segments(per_chunk * B * H * chunks)
        if backward:
            parts = rls.gated_delta_backward(*args, do, d["state"], d["reset"], dlast)
            assert all(torch.equal(x, y) for x, y in zip(parts, whole[1]))
        else:
            o, last = rls.gated_delta(**d)
            assert torch.equal(o, whole[0][0]) and torch.equal(last, whole[0][1])
            state = d["state"].clone()
            o, last = rls.gated_delta(**{**d, "state": state}, last=state)
            assert last is state and torch.equal(state, whole[0][1]) and torch.equal(o, whole[0][0])


@pytest.mark.parametrize("T", [1, 6, 8, 9, 64, 130])
def test_a_sequence_in_pieces(rls, T):
    """Calls that hand the state on, in place, are one call."""
    d = inputs(2, 200, 4, 2, 64, 96, "bf16", 7, True)
    o, last = rls.gated_delta(**d)
    state, version, parts = d["state"].clone(), None, []
    for t in range(0, 200, T):
        part = {n: (x[:, t:t + T] if n in "qkv" else x[:, t:t + T].contiguous()) for n, x in d.items() if n != "state"}
        version = state._version
        parts.append(rls.gated_delta(**part, state=state, last=state)[0])
        assert state._version > version
    close(state, last, 200, 64, 2, "state")
    close(torch.cat(parts, 1).float(), o.float(), 200, 64, 2.0 + 2.0 ** -8 / (8 * UNIT * (264 * 128) ** 0.5), "o")


def test_gates_at_their_ends(rls):
    """Decays of 0 and less than the smallest number, beta 0 and 1, a step that is cut off: what is carried, and the gradients there."""
    for T in (7, 150):
        d = inputs(1, T, 2, 2, 32, 32, "f32", 1)
        d["g"][:, 2, 0], d["g"][:, 3, 1], d["g"][:, 5] = -torch.inf, -90.0, 0.0
        d["beta"][:, 1], d["beta"][:, 4] = 0.0, 1.0
        o, last = rls.gated_delta(**d)
        want, end = loop(*d.values(), 32 ** -0.5)
        close(o, want, T, 32, 1, "o")
        close(last, end, T, 32, 1, "last")
        do, dlast = torch.ones_like(o), torch.ones_like(last)
        got = rls.gated_delta_backward(*(d[n] for n in ("q", "k", "v", "g", "beta")), do, d["state"], None, dlast)
        d["g"] = d["g"].clamp(min=-200.0)                # (the loop's own gradient at -infinity is no number)
        want = gradients(d, do, dlast, 32 ** -0.5)
        for x, y in zip(got, (want[n] for n in ("q", "k", "v", "g", "beta", "state"))):
            close(x, y, T, 32, 2, "gradient")
        assert got[3][0, 2, 0] == 0 and got[3][0, 3, 1] == 0


def test_nothing_passes_a_reset(rls):
    for T in (6, 100):
        d = inputs(2, T, 2, 1, 32, 48, "bf16", 3)
        d["reset"] = torch.zeros(2, T, dtype=torch.bool, device="cuda")
        d["reset"][:, T // 2] = True
        o, last = rls.gated_delta(**d)
        alone, end = rls.gated_delta(**{n: x[:, T // 2:].contiguous() for n, x in d.items() if n not in ("state", "reset")})
        close(last, end, T, 32, 2, "last")
        close(o[:, T // 2:].float(), alone.float(), T, 32, 2 + 2.0 ** -7 / (8 * UNIT * ((T + 64) * 96) ** 0.5), "o")
        zero = d["state"] * 0
        assert torch.equal(rls.gated_delta(**{**d, "state": zero})[1], rls.gated_delta(**{**d, "state": None})[1])


def test_no_steps(rls):
    d = inputs(2, 0, 2, 1, 16, 16, "f32", 1)
    o, last = rls.gated_delta(**d)
    assert o.shape == (2, 0, 2, 16) and torch.equal(last, d["state"])
    assert not rls.gated_delta(**{**d, "state": None})[1].any()
    grads = rls.gated_delta_backward(*(d[n] for n in ("q", "k", "v", "g", "beta")), o, d["state"], None, d["state"])
    assert torch.equal(grads[5], d["state"])


@pytest.mark.parametrize("T", [3, 90])
def test_views(rls, T):
    """Heads out of one projection, steps in the first place, shared rows; written rows lie where they should and nothing else changes."""
    B, H, K, V = 2, 3, 24, 40
    whole = torch.randn(T, B, H * (2 * K + V) + 5, dtype=torch.float32).to(torch.bfloat16).cuda().transpose(0, 1)
    parts = whole[..., 1:1 + H * (2 * K + V)].unflatten(-1, (H, 2 * K + V))
    q, k, v = parts[..., :K] * 0.2, parts[..., K:2 * K], parts[..., 2 * K:]
    k = torch.nn.functional.normalize(k[:, :1].float(), dim=-1).to(torch.bfloat16).expand(B, T, H, K)
    d = inputs(B, T, H, H, K, V, "bf16", 1)
    out = torch.full((B, T, H, V + 3), 5.0, dtype=torch.bfloat16, device="cuda")
    got, last = rls.gated_delta(q, k, v, d["g"], d["beta"], d["state"], out=out[..., 1:1 + V])
    want, end = loop(q, k, v, d["g"], d["beta"], d["state"], None, K ** -0.5)
    close(got, want, T, K, 1, "o")
    close(last, end, T, K, 1, "last")
    assert bool((out[..., 0] == 5).all()) and bool((out[..., 1 + V:] == 5).all())
    do = torch.randn(T, B, H, V, device="cuda").to(torch.bfloat16).transpose(0, 1)
    grads = rls.gated_delta_backward(q, k, v, d["g"], d["beta"], do, d["state"])
    again = rls.gated_delta_backward(q.contiguous(), k.contiguous(), v.contiguous(), d["g"], d["beta"], do.contiguous(), d["state"])
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


def test_autograd(rls):
    d = inputs(2, 40, 4, 2, 32, 32, "f32", 2, True)
    by, by_last = torch.randn(2, 40, 4, 32).cuda(), torch.randn(2, 4, 32, 32).cuda()
    names = ["q", "k", "v", "g", "beta", "state"]
    for which in (names, ["v"], ["g", "beta"], ["state"]):
        for part in ("both", "o", "last"):
            leaves = {n: d[n].clone().requires_grad_() for n in which}
            o, last = rls.gated_delta(**{**d, **leaves})
            value = (o * by).sum() * (part != "last") + (last * by_last).sum() * (part != "o") if part == "both" else (o * by).sum() if part == "o" else (last * by_last).sum()
            got = torch.autograd.grad(value, list(leaves.values()))
            want = gradients(d, by * (part != "last"), by_last * (part != "o"), 32 ** -0.5)
            for n, x in zip(which, got):
                w = want[n].masked_fill(d["reset"][:, :, None] != 0, 0.0) if n == "g" else want[n]
                close(x, w, 40, 32, 2, (n, part))
    with pytest.raises(ValueError):
        rls.gated_delta(**{**d, "q": d["q"].clone().requires_grad_()}, last=d["state"])
    # against differences: along a direction of all inputs (the value is smooth; a step of 2^-8, an error of its third derivative's order and of roundings over it)
    way = {n: torch.randn_like(d[n]) * 0.1 for n in names}
    value = lambda e: (lambda r: (r[0] * by).double().sum() + (r[1] * by_last).double().sum())(rls.gated_delta(**{**d, **{n: d[n] + e * way[n] for n in names}}))     # noqa: E731
    h = 2.0 ** -8
    slope = (value(h) - value(-h)) / (2 * h)
    got = rls.gated_delta_backward(*(d[n] for n in names[:5]), by, d["state"], d["reset"], by_last)
    sum_of = sum((x.double() * way[n].double()).sum() for n, x in zip(names, got))
    size = sum((x.double() * way[n].double()).square().sum() for n, x in zip(names, got)) ** 0.5
    assert abs(float(slope - sum_of)) < 0.02 * float(size) + 0.02 * abs(float(sum_of))


def test_graph_and_streams(rls):
    shapes = [(2, 1, 4, 2, 64, 64), (2, 150, 4, 2, 64, 64)]
    for shape in shapes:
        B, T, H, HK, K, V = shape
        d = inputs(*shape, "bf16", 1, True)
        do = torch.randn(B, T, H, V).to(torch.bfloat16).cuda()
        ws = torch.empty(max(rls.gated_delta_workspace_bytes(*shape, backward=b) for b in (False, True)) + 256, dtype=torch.uint8, device="cuda")

        def both(d, ws):
            args = [d[n] for n in ("q", "k", "v", "g", "beta")]
            return (*rls.gated_delta(**d, workspace=ws), *rls.gated_delta_backward(*args, do, d["state"], d["reset"], workspace=ws))
        both(d, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = both(d, ws)
        for seed in range(4):
            for n, x in inputs(*shape, "bf16", 10 + seed, True).items():
                d[n].copy_(x)
            want = both(d, None)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want)), seed
        ds = [inputs(*shape, "bf16", 20 + i, True) for i in range(3)]
        want = [both(x, None) for x in ds]
        torch.cuda.synchronize()
        streams, results = [torch.cuda.Stream() for _ in ds], []
        for st, x in zip(streams, ds):
            with torch.cuda.stream(st):
                results.append([both(x, None) for _ in range(3)][-1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for r, w in zip(results, want) for x, y in zip(r, w))


@pytest.mark.parametrize("T", [4, 100])
def test_sequences_past_32_bits(rls, T):
    """Sequences whose rows begin more than 2^31 elements after each other's."""
    H, K = 2, 64
    d = inputs(2, T, H, H, K, K, "bf16", 5)
    far = torch.empty((1 << 31) + 3 * T * H * K, dtype=torch.bfloat16, device="cuda")
    views = {n: far[i * T * H * K:].as_strided((2, T, H, K), (1 << 31, H * K, K, 1)) for i, n in enumerate("qkv")}
    for n, x in views.items():
        x.copy_(d[n])
    o, last = rls.gated_delta(**{**d, **views})
    want, end = rls.gated_delta(**d)
    assert torch.equal(o, want) and torch.equal(last, end)
    rest = d["g"], d["beta"], o, d["state"], None, last
    for x, y in zip(rls.gated_delta_backward(*views.values(), *rest), rls.gated_delta_backward(d["q"], d["k"], d["v"], *rest)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("T", [2, 70, 300])
def test_the_states_gradient_in_place(rls, short_segments, T):
    """Through the C ABI: dstate written where dlast was, with one segment and with several; without dlast or dstate at all."""
    B, H, K, V = 2, 2, 32, 48
    d = inputs(B, T, H, 1, K, V, "f32", 9, True)
    do, dlast = torch.randn(B, T, H, V, device="cuda"), torch.randn(B, H, K, V, device="cuda")
    args = [d[n] for n in ("q", "k", "v", "g", "beta")]
    want = rls.gated_delta_backward(*args, do, d["state"], d["reset"], dlast)
    none = rls.gated_delta_backward(*args, do, d["state"], d["reset"])
    for segment in (-1, 0):
        short_segments(segment)
        shape = rls._DeltaShape(B, T, H, 1, K, V, 0, K ** -0.5)
        ws = torch.empty(rls.gated_delta_workspace_bytes(B, T, H, 1, K, V, True) + 256, dtype=torch.uint8, device="cuda")
        base = ws.data_ptr() + -ws.data_ptr() % 256
        for by, to, expected in ((dlast.clone(), "same", want), (None, None, none)):
            out = [torch.empty_like(x) for x in want[:5]]
            held, at = rls._heads(torch.float32, *((x, x.shape, "x") for x in (d["q"], d["k"], d["v"], do, out[0], out[1], out[2])))
            rc = rls.lib().rls_gated_delta_backward(ctypes.byref(shape), at[0], at[1], at[2], d["g"].data_ptr(), d["beta"].data_ptr(), d["state"].data_ptr(),
                                                    d["reset"].data_ptr(), at[3], 0 if by is None else by.data_ptr(), at[4], at[5], at[6], out[3].data_ptr(),
                                                    out[4].data_ptr(), by.data_ptr() if to else 0, base, ws.numel() - 256,
                                                    torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            assert all(torch.equal(x, y) for x, y in zip(out, expected))
            assert by is None or torch.equal(by, want[5])
