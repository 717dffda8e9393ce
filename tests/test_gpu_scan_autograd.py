"""rls.linear_scan inside autograd, and what autograd is told about tensors that the library changes in place.

Gradients of sequences of at most 60 steps with gates below 1, to 64 roundings of the largest one in the type they are held in."""
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


def loop(a, b, h0, reset, reverse):
    """The same layer step by step."""
    B, T, C = b.shape
    s = torch.zeros(B, C, dtype=b.dtype, device=b.device) if h0 is None else h0
    out = [None] * T
    for t in reversed(range(T)) if reverse else range(T):
        carried = a[:, t] * s
        s = (carried if reset is None else torch.where(reset[:, t, None] != 0, torch.zeros_like(carried), carried)) + b[:, t]
        out[t] = s
    return torch.stack(out, 1), s


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("B,T,C", [(3, 1, 5), (2, 50, 7), (4, 60, 130), (3, 40, 1)])
@pytest.mark.parametrize("which", ["all", "gate", "input", "state", "states only", "last only", "reset", "shared gate", "no state"])
def test_gradients(rls, B, T, C, which, reverse):
    gen = torch.Generator().manual_seed(T + C)
    draw = lambda *shape: torch.randn(*shape, generator=gen).cuda()      # noqa: E731
    gate = torch.sigmoid(draw(1, 1, C) if which == "shared gate" else draw(B, T, C))
    inputs = {"a": gate, "b": draw(B, T, C), "h0": draw(B, C)}
    wanted = {"gate": ["a"], "input": ["b"], "state": ["h0"], "no state": ["a", "b"]}.get(which, ["a", "b", "h0"])
    for name in wanted:
        inputs[name].requires_grad_()
    reset = (torch.rand(B, T, generator=gen) < 0.2).to(torch.uint8).cuda() if which == "reset" else None
    by_h, by_last = draw(B, T, C), draw(B, C)

    def loss(scan, kind):
        a, b, h0 = (inputs[k].to(kind) for k in ("a", "b", "h0"))
        h, last = scan(a.expand(B, T, C), b, None if which == "no state" else h0, reset, reverse)
        if which == "states only":
            return (h * by_h).sum()
        if which == "last only":
            return (last * by_last).sum()
        return (h * by_h).sum() + (last * by_last).sum()

    leaves = [inputs[name] for name in wanted]
    got = torch.autograd.grad(loss(rls.linear_scan, torch.float32), leaves)
    want = torch.autograd.grad(loss(loop, torch.float64), leaves)
    for x, y, name in zip(got, want, wanted):
        terms = B * T if which == "shared gate" and name == "a" else 1       # (summed by autograd, in fp32 here)
        assert (x.double() - y.double()).abs().max() <= terms * 2.0 ** -18 * y.abs().max(), name


def test_in_a_type_of_16_bits(rls):
    """Gradients of every element stay in the types of their inputs; nothing is differentiated under no_grad."""
    gen = torch.Generator().manual_seed(1)
    a = torch.sigmoid(torch.randn(2, 30, 9, generator=gen)).cuda().requires_grad_()
    b = torch.randn(2, 30, 9, generator=gen).cuda().bfloat16().requires_grad_()
    h, last = rls.linear_scan(a, b)
    assert h.dtype == torch.bfloat16 and last.dtype == torch.float32 and h.requires_grad and last.requires_grad
    da, db = torch.autograd.grad(h.float().sum() + last.sum(), (a, b))
    ra, rb, _ = rls.linear_scan_backward(a.detach(), h.detach(), torch.ones_like(h).detach(), None, None, torch.ones(2, 9).cuda())
    assert da.dtype == torch.float32 and db.dtype == torch.bfloat16 and torch.equal(da, ra) and torch.equal(db, rb)
    with torch.no_grad():
        h, last = rls.linear_scan(a, b, out=torch.empty_like(b), last=torch.empty(2, 9).cuda())
    assert not h.requires_grad and not last.requires_grad
    for given in ({"out": torch.empty_like(b)}, {"last": torch.empty(2, 9).cuda()}):
        with pytest.raises(ValueError):
            rls.linear_scan(a, b, **given)


def test_tensors_changed_in_place_are_known_to_autograd(rls):
    """A graph that saved a tensor which a call has changed since then raises, as after torch's own in-place operations."""
    state = torch.ones(2, 3).cuda()
    x = torch.ones(2, 3).cuda().requires_grad_()
    y = (x * state).sum()
    rls.linear_scan(torch.ones(2, 1, 3).cuda(), torch.ones(2, 1, 3).cuda(), state, last=state)
    with pytest.raises(RuntimeError):
        y.backward()
    p = torch.ones(5).cuda().requires_grad_()
    opt = rls.AdamW([p.detach()])
    y = (p * p).sum()
    opt.step([torch.ones(5).cuda()])
    with pytest.raises(RuntimeError):
        y.backward()
    out = torch.zeros(2, 4, 3).cuda()
    y = (x[:, None] * out).sum()
    rls.linear_scan(torch.ones(2, 4, 3).cuda(), torch.ones(2, 4, 3).cuda(), out=out)
    with pytest.raises(RuntimeError):
        y.backward()
    # tensors of inference mode have no such counter
    with torch.inference_mode():
        q, s = torch.ones(5).cuda(), torch.ones(2, 3).cuda()
        rls.AdamW([q]).step([torch.ones(5).cuda()])
        rls.linear_scan(torch.ones(2, 1, 3).cuda(), torch.ones(2, 1, 3).cuda(), s, last=s)
    assert (q < 1).all() and (s == 2).all()
