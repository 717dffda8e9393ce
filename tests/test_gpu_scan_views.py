"""Linear scans on views of one buffer: side by side and between each other's rows they are served, over each other they are turned down."""
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


def apart(t):
    """The same view of a buffer of its own (the strides decide which kernel takes a call of one channel, and so its rounding)."""
    return torch.empty_strided(t.shape, t.stride(), device="cuda").copy_(t)


@pytest.mark.parametrize("B,T,C", [(2, 5, 7), (3, 300, 65), (1, 6000, 40), (2, 700, 1), (64, 1, 33)])
def test_records_of_gate_input_and_output(rls, B, T, C):
    gen = torch.Generator().manual_seed(T)
    for turned in (False, True):
        whole = torch.empty((T, B, 3, C) if turned else (B, T, 3, C), device="cuda")
        a, b, out = (v.transpose(0, 1) if turned else v for v in whole.unbind(2))
        a.copy_(torch.sigmoid(torch.randn(B, T, C, generator=gen) + 2.0))
        b.copy_(torch.randn(B, T, C, generator=gen))
        want, want_last = rls.linear_scan(apart(a), apart(b), out=apart(out))
        h, last = rls.linear_scan(a, b, out=out)
        assert h is out and torch.equal(h, want) and torch.equal(last, want_last)
        shared = a[:1].expand(B, T, C)
        h, last = rls.linear_scan(shared, b, out=out)
        assert torch.equal(h, rls.linear_scan(apart(a)[:1].expand(B, T, C), apart(b), out=apart(out))[0])


def test_over_an_input(rls):
    a, b = torch.full((2, 30, 8), 0.5).cuda(), torch.ones(2, 30, 8).cuda()
    for out in (a, b):
        with pytest.raises(rls.RlsError):
            rls.linear_scan(a, b, out=out)
    wide = torch.ones(2, 30, 12).cuda()
    with pytest.raises(rls.RlsError):
        rls.linear_scan(a, wide[:, :, :8], out=wide[:, :, 4:])
    assert (a == 0.5).all() and (b == 1).all() and (wide == 1).all()
