"""rls.gated_delta: what lies behind a reset, or a gate that keeps nothing, does not reach what lies before it, and the other way round.

Tolerances as in test_gpu_delta: errors of a sequence by itself, relative to its own largest value."""
import pytest
import torch

from tests.test_gpu_delta import close, gradients, inputs, rls              # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,cut", [(64, 63), (60, 7), (100, 40), (200, 128), (200, 150)])
def test_gradients_before_a_cut_beside_large_ones_behind_it(rls, T, cut, kind):     # noqa: F811
    """Gradients behind the cut 2^20 times as large: those by the gates before it keep their digits."""
    shape = B, _, H, HK, K, V = 2, T, 4, 2, 48, 40
    for gate in (False, True):
        d = inputs(*shape, kind, T + cut)
        if gate:
            d["g"][:, cut] = -torch.inf
        else:
            d["reset"] = torch.zeros(B, T, dtype=torch.uint8, device="cuda")
            d["reset"][:, cut] = 1
        do = torch.randn(B, T, H, V, generator=torch.Generator().manual_seed(cut)).cuda()
        do[:, cut:] *= 2.0 ** 20 if kind == "f32" else 2.0 ** 12
        do = do.to(d["v"].dtype)
        names = ("q", "k", "v", "g", "beta")
        got = dict(zip(names + ("state",), rls.gated_delta_backward(*(d[n] for n in names), do, d["state"], d["reset"], scale=0.3)))
        alone = {n: (None if d[n] is None else d[n] if n == "state" else d[n][:, :cut].contiguous()) for n in names + ("state", "reset")}
        want = gradients(alone, do[:, :cut], None, 0.3)
        terms = (alone["beta"] * want["beta"]).abs().max()
        for n, w in want.items():
            close(got[n] if n == "state" else got[n][:, :cut], w, T, K, 2, (n, gate), terms if n == "g" else 0.0)


def by_steps(d, scale):
    """The recurrence in 64 bits, a cut (a reset, or a gate below -87) taken as such: nothing of the state before it counts."""
    q, k, v, g, beta = (d[n].double() for n in ("q", "k", "v", "g", "beta"))
    group = v.shape[2] // q.shape[2]
    q, k = q.repeat_interleave(group, 2), k.repeat_interleave(group, 2)
    B, T, H, V = v.shape
    s, out = torch.zeros(B, H, q.shape[3], V, dtype=torch.float64, device=v.device) if d["state"] is None else d["state"].double(), []
    for t in range(T):
        cut = g[:, t] < -87.0
        if d["reset"] is not None:
            cut = cut | (d["reset"][:, t, None] != 0)
        s = torch.where(cut[:, :, None, None], 0.0, torch.exp(g[:, t])[:, :, None, None] * s)
        y = v[:, t] - (s * k[:, t, :, :, None]).sum(2)
        s = s + k[:, t, :, :, None] * (beta[:, t, :, None] * y)[:, :, None]
        out.append(scale * (s * q[:, t, :, :, None]).sum(2))
    return torch.stack(out, 1), s


def same_where_finite(got, want, T, K, twice, what):
    finite = want.isfinite() & (want.abs() < torch.finfo(got.dtype).max)
    assert torch.equal(got.isfinite(), finite), (what, int((got.isfinite() != finite).sum()))
    close(torch.where(finite, got, 0.0), torch.where(finite, want, 0.0), T, K, twice, what)


BAD = [("q", 0), ("k", 0), ("v", 0), ("g", 0), ("beta", 0), ("q", 1), ("k", 1), ("v", 1), ("beta", 1), ("state", 0), ("state", 1)]
# steps, cuts, the step of the number that is not finite
PLACES = [(5, (3,), 1), (5, (3,), 3), (40, (10, 30), 12), (64, (10, 63), 40), (100, (70,), 64), (100, (20, 80), 20), (200, (64, 128, 140), 100), (200, (64, 128, 140), 150)]


@pytest.fixture
def cut_segments(rls):                                                           # noqa: F811
    import ctypes
    set_bytes = rls.lib().rls_delta_segment_bytes
    set_bytes.argtypes = [ctypes.c_int64]
    yield lambda n: set_bytes(n)
    set_bytes(-1)


def with_cuts(d, cuts, gates):
    d["reset"] = torch.zeros(d["v"].shape[:2], dtype=torch.uint8, device="cuda")
    for i, t in enumerate(cuts):
        if gates and i % 2 == 0:
            d["g"][:, t] = -torch.inf
        else:
            d["reset"][:, t] = 1


def put_bad(d, name, at, kind):
    """One number that is not finite: of the second sequence, at its second head (the first, of keys)."""
    x = torch.inf if kind else torch.nan
    if name == "state":
        d["state"][1, 1, 3, 2] = x
    elif name in ("g", "beta"):
        d[name][1, at, 1] = x
    else:
        d[name][1, at, 0 if name in "qk" else 1, 2] = x


@pytest.mark.parametrize("kind,K,V", [("f32", 32, 40), ("bf16", 48, 16), ("f16", 64, 33), ("bf16", 128, 130), ("f32", 128, 64)])
@pytest.mark.parametrize("T,cuts,at", PLACES)
def test_numbers_that_are_not_finite(rls, cut_segments, T, cuts, at, kind, K, V):              # noqa: F811
    """What one makes not finite in the recurrence step by step, that and nothing else: neither what lies before it nor, behind the next cut, what follows."""
    for i, (name, what) in enumerate(BAD):
        d = inputs(2, T, 4, 2, K, V, kind, T + i)
        with_cuts(d, cuts, i % 2)
        if name == "g" and at in cuts:
            continue                                     # (a gate that is reset is not looked at)
        put_bad(d, name, at, what)
        want, end = by_steps(d, K ** -0.5)
        assert bool(end.isfinite().any()) and (not bool(want.isfinite().all()) or (name == "state" and cuts[0] == 0))
        for segment in (-1, 0):
            cut_segments(segment)
            state = d["state"].clone()
            o, last = rls.gated_delta(**{**d, "state": state}, last=state)
            same_where_finite(o, want, T, K, 1, (name, what, "o"))
            same_where_finite(last, end, T, K, 1, (name, what, "last"))


@pytest.mark.parametrize("T", [4, 30, 70, 130])
def test_padding_behind_the_last_step(rls, T):                                   # noqa: F811
    """Steps behind the end of a sequence hold anything: what lies before them is as without them."""
    d = inputs(3, T, 4, 2, 32, 48, "bf16", T)
    ends = [T, T - 3, max(1, T // 2)]
    whole = by_steps({**d, "reset": None}, 32 ** -0.5)[0]
    for b, end in enumerate(ends):
        for n in ("q", "k", "v", "g", "beta"):
            d[n][b, end:] = torch.nan
    o, _ = rls.gated_delta(**d)
    for b, end in enumerate(ends):
        close(o[b, :end], whole[b, :end], T, 32, 1, b)
    assert rls.gated_delta(**{**d, "reset": None})[1][0].isfinite().all()


def test_decays_beyond_the_largest_number(rls):                                  # noqa: F811
    """Gates above 0 whose product over some steps is no number in fp32, while the state always is."""
    d = inputs(2, 100, 2, 2, 32, 32, "f32", 3)
    d["state"] *= 1e-30
    d["g"][:, :30], d["g"][:, 30:60], d["g"][:, 60:] = 4.0, -4.0, 0.0
    d["beta"][:, :70] = 0.0
    o, last = rls.gated_delta(**d)
    want, end = by_steps(d, 32 ** -0.5)
    close(o, want, 100, 32, 1, "o")
    close(last, end, 100, 32, 1, "last")


BAD_BACK = BAD + [("do", 0), ("do", 1), ("dlast", 0), ("dlast", 1)]


@pytest.mark.parametrize("kind,K,V", [("f32", 32, 40), ("bf16", 48, 16), ("f16", 64, 33), ("bf16", 128, 130), ("f32", 128, 64)])
@pytest.mark.parametrize("T,cuts,at", PLACES)
def test_gradients_of_numbers_that_are_not_finite(rls, cut_segments, T, cuts, at, kind, K, V):     # noqa: F811
    """Between two cuts one spoils the gradients of its head; those between other cuts, and of other heads and sequences, are as if it were not there."""
    B, H, HK = 2, 4, 2
    names = ("q", "k", "v", "g", "beta")
    gen = torch.Generator().manual_seed(T)
    for i, (name, what) in enumerate(BAD_BACK):
        d = inputs(B, T, H, HK, K, V, kind, T + i)
        with_cuts(d, cuts, i % 2)
        if name == "g" and at in cuts:
            continue
        do, dlast = torch.randn(B, T, H, V, generator=gen).to(d["v"].dtype).cuda(), torch.randn(B, H, K, V, generator=gen).cuda()
        edges = [0, *cuts, T]
        want = []
        for p, (a, e) in enumerate(zip(edges, edges[1:])):
            part = {n: d[n][:, a:e].contiguous() for n in names}
            part["g"][:, 0] = 0.0 if p else part["g"][:, 0]                        # (what a cut has is not looked at)
            part |= {"state": d["state"] if p == 0 else torch.zeros_like(d["state"]), "reset": None}
            want.append(gradients(part, do[:, a:e], dlast if e == T else None, 0.3))
            if p:
                want[p]["g"][:, 0] = 0.0
        if name == "do":
            do[1, at, 1, 2] = torch.inf if what else torch.nan
        elif name == "dlast":
            dlast[1, 1, 3, 2] = torch.inf if what else torch.nan
        else:
            put_bad(d, name, at, what)
        spoilt = 0 if name == "state" else len(cuts) if name == "dlast" else max(p for p, a in enumerate(edges[:-1]) if a <= at)
        for segment in (-1, 0):
            cut_segments(segment)
            got = dict(zip(names + ("state",), rls.gated_delta_backward(*(d[n] for n in names), do, d["state"], d["reset"], dlast, scale=0.3)))
            assert not all(bool(x.isfinite().all()) for x in got.values())
            for p, (a, e) in enumerate(zip(edges, edges[1:])):
                for n in names + (("state",) if p == 0 else ()):
                    x, w = got[n] if n == "state" else got[n][:, a:e], want[p][n]
                    # heads by themselves: those that the bad number's does not reach, and all where the part is another one
                    reached = torch.zeros_like(w, dtype=torch.bool)
                    if p == spoilt and name in "qk":     # (both heads that share the key)
                        (reached[1, 0:2] if n == "state" else reached[1, :, 0:1] if n in "qk" else reached[1, :, 0:2])[:] = True
                    elif p == spoilt:
                        (reached[1, 1:2] if n == "state" else reached[1, :, 0:1] if n in "qk" else reached[1, :, 1:2])[:] = True
                    terms = (d["beta"][:, a:e].nan_to_num(1.0, 1.0) * want[p]["beta"]).abs().max()
                    close(torch.where(reached, 0.0, x.double()).to(x.dtype), torch.where(reached, 0.0, w), T, K, 2, (name, what, p, n, segment), terms if n == "g" else 0.0)


@pytest.mark.parametrize("T", [6, 40])
def test_answers_beyond_the_largest_number_before_a_cut(rls, T):                 # noqa: F811
    """A finite state whose product with a query is not: what lies behind the cut is answered without it."""
    d = inputs(2, T, 2, 1, 32, 16, "f32", T)
    with_cuts(d, (4,), False)
    d["state"] = torch.full_like(d["state"], 3e38)
    d["q"] = torch.full_like(d["q"], 32 ** -0.5)                                   # q . S is 5.7 times a row's entry
    d["k"].zero_()
    d["k"][..., 3] = 1.0
    d["g"][:, :4] = 0.0
    d["beta"][:, :4] = 0.0
    o, last = rls.gated_delta(**d, scale=1.0)
    want, end = by_steps(d, 1.0)
    assert not bool(o[:, :4].isfinite().any())
    close(o[:, 4:], want[:, 4:], T, 32, 1, "o")
    close(last, end, T, 32, 1, "last")
