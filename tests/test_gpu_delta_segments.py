"""rls.gated_delta in segments of several chunks, as with long sequences of many heads: the same bits as in one."""
import ctypes

import pytest
import torch

from tests.test_gpu_delta import TYPES, close, gradients, inputs, loop, rls   # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture
def segments(rls):                                                               # noqa: F811
    """segments(shape, kind, backward, chunks): calls of that shape take segments of so many chunks, which is asserted."""
    L = rls.lib()
    L.rls_delta_segment_bytes.argtypes = [ctypes.c_int64]
    L.rls_delta_segment_chunks.restype = ctypes.c_int64
    L.rls_delta_segment_chunks.argtypes = [ctypes.c_void_p, ctypes.c_int32]

    def cut(shape, kind, backward, chunks):
        B, T, H, HK, K, V = shape
        s = rls._DeltaShape(B, T, H, HK, K, V, list(TYPES).index(kind), 1.0)
        lo, hi = 0, 1 << 40                              # the fewest bytes with which a segment has as many
        while lo < hi:
            at = (lo + hi) // 2
            L.rls_delta_segment_bytes(at)
            if L.rls_delta_segment_chunks(ctypes.byref(s), backward) >= chunks:
                hi = at
            else:
                lo = at + 1
        L.rls_delta_segment_bytes(hi)
        assert L.rls_delta_segment_chunks(ctypes.byref(s), backward) == chunks
    yield cut
    L.rls_delta_segment_bytes(-1)


# 8 chunks, the last of 2 steps: in segments of 3 and 2 (three of them 3, 3 and 2, the last one short in both ways)
@pytest.mark.parametrize("shape,kind", [((2, 450, 4, 2, 64, 64), "f32"), ((1, 450, 2, 2, 128, 128), "bf16"), ((2, 450, 6, 2, 128, 72), "bf16"), ((1, 450, 2, 1, 128, 40), "f32"),
                                        ((2, 450, 4, 2, 33, 130), "f16"), ((1, 450, 2, 2, 128, 64), "f16"), ((3, 330, 2, 1, 20, 24), "bf16")])
@pytest.mark.parametrize("chunks", [1, 2, 3])
def test_segments_of_several_chunks(rls, segments, shape, kind, chunks):         # noqa: F811
    B, T, H, HK, K, V = shape
    d = inputs(*shape, kind, 3, True)
    gen = torch.Generator().manual_seed(1)
    do, dlast = torch.randn(B, T, H, V, generator=gen).to(TYPES[kind]).cuda(), torch.randn(B, H, K, V, generator=gen).cuda()
    names = ("q", "k", "v", "g", "beta")
    args = [d[n] for n in names]
    o, last = rls.gated_delta(**d)
    whole = rls.gated_delta_backward(*args, do, d["state"], d["reset"], dlast)
    segments(shape, kind, 0, chunks)
    state = d["state"].clone()
    for got in (rls.gated_delta(**d), rls.gated_delta(**{**d, "state": state}, last=state)):
        assert torch.equal(got[0], o) and torch.equal(got[1], last)
    close(got[0], loop(*d.values(), K ** -0.5)[0], T, K, 1, "o")
    segments(shape, kind, 1, chunks)
    parts = rls.gated_delta_backward(*args, do, d["state"], d["reset"], dlast)
    assert all(torch.equal(x, y) for x, y in zip(parts, whole))
    if chunks == 3:
        want = gradients(d, do, dlast, K ** -0.5)
        want["g"] = want["g"].masked_fill(d["reset"][:, :, None] != 0, 0.0)
        terms = (d["beta"] * want["beta"]).abs().max()
        for n, x in zip(names + ("state",), parts):
            close(x, want[n], T, K, 2, n, terms if n == "g" else 0.0)
