"""The state of a linear scan in place: h_last in h0's memory and dh0 in dh_last's, over sequences that one workgroup takes by itself.

The last steps lie with other waves than the first ones, which must all have read the state before it is written over: the same bits as with the
two apart."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = [(2, 20, 130), (2, 40, 130), (2, 64, 128), (2, 100, 33), (1, 100, 130), (2, 128, 130), (64, 127, 516), (3, 200, 5), (3, 2000, 1), (1, 3000, 1), (200, 4096, 1)]


@pytest.fixture(scope="module")
def rls():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_1905_12799_amd import binding
    binding.lib()
    return binding


def make(B, T, C, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    draw = lambda *shape: torch.randn(*shape, generator=gen)     # noqa: E731
    a = torch.sigmoid(draw(B, T, C) + 2.0)
    return a.cuda(), draw(B, T, C).to(dtype).cuda(), draw(B, T, C).to(dtype).cuda(), draw(B, C).cuda()


@pytest.mark.parametrize("B,T,C", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_forward(rls, B, T, C, dtype):
    a, b, _, h0 = make(B, T, C, dtype, T)
    for reverse in (False, True):
        want_h, want = rls.linear_scan(a, b, h0, reverse=reverse)
        for _ in range(5):
            state = h0.clone()
            h, last = rls.linear_scan(a, b, state, reverse=reverse, last=state)
            assert last is state and torch.equal(h, want_h) and torch.equal(last, want)


@pytest.mark.parametrize("B,T,C", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward(rls, B, T, C, dtype):
    a, h, dh, h0 = make(B, T, C, dtype, T + 1)
    dlast = h0 * 0.5 + 1.0
    for reverse in (False, True):
        want_da, want_db, want = rls.linear_scan_backward(a, h, dh, h0, dh_last=dlast, reverse=reverse)
        kind = 0 if dtype == torch.float32 else 1
        shape = rls._ScanShape(B, T, C, kind, 0, int(reverse))
        seq = lambda t: ctypes.byref(rls._Sequence(t.data_ptr(), T * C, C))      # noqa: E731
        need = rls.linear_scan_workspace_bytes(B, T, C)
        space = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
        base = (space.data_ptr() + 255) // 256 * 256
        for _ in range(5):
            da, db, state = torch.empty_like(a), torch.empty_like(h), dlast.clone()
            rc = rls.lib().rls_linear_scan_backward(ctypes.byref(shape), seq(a), seq(h), seq(dh), h0.data_ptr(), None, state.data_ptr(), seq(da), seq(db),
                                                    state.data_ptr(), base, need, torch.cuda.current_stream().cuda_stream)
            assert rc == 0
            assert torch.equal(da, want_da) and torch.equal(db, want_db) and torch.equal(state, want)
