"""The tensors that an AdamW optimizer holds: other ones in its lists, other memory behind them, and what it turns down.

Where a tensor is replaced, its old memory is kept by the test and must stay as it was."""
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


def tensors(sizes, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn(n, generator=gen).to(dtype).cuda() for n in sizes]


SIZES = [1, 300, 5000]
LISTS = ["params", "exp_avg", "exp_avg_sq", "master", "exp_avg_scale", "exp_avg_sq_scale"]


def twins(rls, dtype, bits, master):
    """Two optimizers in the same state, a step done."""
    pair = []
    for _ in range(2):
        opt = rls.AdamW(tensors(SIZES, dtype, 1), state_bits=bits, master=master, seed=5)
        opt.step(tensors(SIZES, dtype, 2))
        pair.append(opt)
    return pair


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip((t for x in a._lists() for t in x), (t for x in b._lists() for t in x)))


@pytest.mark.parametrize("way", ["list", "data", "storage"])
@pytest.mark.parametrize("dtype,bits,master", [(torch.float32, 32, False), (torch.bfloat16, 32, True), (torch.bfloat16, 8, True), (torch.float16, 8, False)])
def test_replaced_tensors_count_from_the_next_step_on(rls, dtype, bits, master, way):
    a, b = twins(rls, dtype, bits, master)
    old, kept = [], []
    for name in LISTS:
        lists = getattr(a, name)
        for i in range(len(lists) if lists is not None else 0):
            t = lists[i]
            old.append(t.detach())
            kept.append(t.clone())
            if way == "list":
                lists[i] = t.clone()
            elif way == "data":
                lists[i].data = t.clone()
            else:
                lists[i].set_(t.clone())
    if way == "storage":                                     # (set_ moves the aliases too: nothing is left of the old memory)
        old = kept
    for opt in (a, b):
        opt.step(tensors(SIZES, dtype, 3))
    assert same(a, b) and all(torch.equal(x, y) for x, y in zip(old, kept))
    assert not any(torch.equal(x, y) for x, y in zip(a.params, tensors(SIZES, dtype, 1)))


def test_memory_that_was_let_go_is_not_written(rls):
    """A parameter moves to other memory and the old one becomes another tensor's."""
    p = torch.ones(1 << 20, device="cuda")
    opt = rls.AdamW([p])
    grad = torch.ones(1 << 20, device="cuda")
    opt.step([grad])
    p.data = torch.full((1 << 20,), 2.0, device="cuda")
    others = [torch.zeros(1 << 20, device="cuda") for _ in range(8)]
    opt.step([grad], lr=0.5, weight_decay=0.0)
    assert all((t == 0).all() for t in others) and (p < 2.0).all() and (p > 1.0).all()


def test_another_size_or_type_is_turned_down_then_too(rls):
    for change in (lambda o: o.exp_avg.__setitem__(0, torch.zeros(299).cuda()), lambda o: o.exp_avg.__setitem__(0, torch.zeros(300).double().cuda()),
                   lambda o: o.exp_avg_sq.__setitem__(0, torch.zeros(300)), lambda o: o.exp_avg_sq.pop(), lambda o: o.params.append(torch.ones(3).cuda()),
                   lambda o: o.params[0].set_(torch.ones(300, 2).cuda()[:, 0]), lambda o: o.exp_avg.__setitem__(0, o.exp_avg_sq[0])):
        opt = rls.AdamW([torch.ones(300).cuda()])
        opt.step([torch.ones(300).cuda()])
        change(opt)
        for _ in range(2):
            with pytest.raises(ValueError):
                opt.step([torch.ones(300).cuda()] * len(opt.params))
        assert opt.step_count == 1


def test_overlapping_tensors_are_turned_down(rls):
    whole = torch.zeros(1000).cuda()
    for params in ([whole, whole], [whole[:600], whole[599:]]):
        with pytest.raises(ValueError):
            rls.AdamW(params)
    with pytest.raises(ValueError):
        rls.AdamW([whole], exp_avg=[whole])
    opt = rls.AdamW([whole[:600], whole[600:], whole[:0], whole[5:5]])
    opt.step([torch.ones(600).cuda(), torch.ones(400).cuda(), torch.ones(0).cuda(), torch.ones(0).cuda()])
    assert (whole < 0).all()


def test_a_recorded_step_keeps_its_tensors(rls):
    """A step in a graph, after a tensor was replaced: replays go on from the new one."""
    p = torch.ones(3000).cuda()
    opt = rls.AdamW([p])
    grad = torch.ones(3000).cuda()
    opt.step([grad])
    opt.exp_avg[0] = torch.full((3000,), 0.25).cuda()
    opt.step([grad])
    twin = rls.AdamW([p.clone()], exp_avg=[opt.exp_avg[0].clone()], exp_avg_sq=[opt.exp_avg_sq[0].clone()], step=2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step([grad])
    for _ in range(3):
        twin.step_count = 2
        twin.step([grad])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p, twin.params[0]) and torch.equal(opt.exp_avg[0], twin.exp_avg[0])
