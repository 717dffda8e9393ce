"""Linear scans on several streams at once: tiles wait for tiles of their own call while those of others hold compute units."""
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


def test_calls_side_by_side(rls):
    """Long sequences, one of them with gates whose products are out of range (its tiles wait for the states before them): the bits that each gives alone."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")      # noqa: E731
    cases = []
    for B, T, C in ((1, 30000, 512), (64, 50000, 1), (2, 20000, 130)):
        cases.append((torch.sigmoid(draw(B, T, C) + 8.0), draw(B, T, C)))
    wild = torch.tensor([2.0 ** 100, 2.0 ** 100, 2.0 ** -100, 2.0 ** -100], device="cuda").repeat(2500)[None, :, None].expand(4, 10000, 64).contiguous()
    cases.append((wild, torch.zeros(4, 10000, 64, device="cuda")))
    h0 = [torch.full((b.shape[0], b.shape[2]), 2.0 ** -110, device="cuda") for _, b in cases]
    want = [rls.linear_scan(a, b, s) for (a, b), s in zip(cases, h0)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for (a, b), s, stream in zip(cases, h0, streams):
            with torch.cuda.stream(stream):
                got.append(rls.linear_scan(a, b, s))
    torch.cuda.synchronize()
    for k, (h, last) in enumerate(got):
        assert torch.equal(h, want[k % len(cases)][0]) and torch.equal(last, want[k % len(cases)][1]), k
    assert torch.isfinite(want[-1][0]).all()
