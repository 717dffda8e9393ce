"""Arrays of a linear scan that lie in each other: found before anything is enqueued (no GPU needed), and views between each other's rows are not."""
import ctypes
import random

import pytest

from paper_1905_12799_amd import binding

F32, BF16 = 0, 1
SHAPE = -3
SIZE = {F32: 4, BF16: 2}


@pytest.fixture(scope="module")
def L():
    L = binding.lib()
    L.rls_scan_overlap.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32]
    return L


def covered(shape, q, kind):
    B, T, C = shape
    at, batch, step = q
    k = SIZE[kind]
    return {at + (n * batch + t * step) * k + byte for n in range(B) for t in range(T) for byte in range(C * k)}


def distances(shape, q, kind):
    """Distances that stay once repeated rows and rows that touch are taken together."""
    B, T, C = shape
    _, batch, step = q
    k, width, out = SIZE[kind], C * SIZE[kind], set()
    for count, apart in sorted([(T, step * k), (B, batch * k)], key=lambda d: d[1]):
        if count == 1 or apart == 0:
            continue
        if not out and apart <= width:
            width += (count - 1) * apart
        else:
            out.add(apart)
    return out


def ask(L, shape, x, kx, y, ky):
    s = binding._ScanShape(*shape, kx, F32, 0)
    return L.rls_scan_overlap(ctypes.byref(s), ctypes.byref(binding._Sequence(*x)), kx, ctypes.byref(binding._Sequence(*y)), ky)


def test_against_every_byte(L):
    rng = random.Random(12799)
    seen = {0: 0, 1: 0}
    for _ in range(6000):
        shape = (rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 4))
        ld = rng.randint(shape[2], 12)
        strides = [(shape[1] * ld, ld), (ld, shape[0] * ld), (0, ld), (ld * shape[1], 0), (0, 0), (shape[1] * ld + rng.randint(0, 9), ld), (1, 2), (3, 1)]
        (kx, ky), x, y = rng.choices([F32, BF16], k=2), rng.choice(strides), rng.choice(strides[:3] if rng.random() < 0.6 else strides)
        if rng.random() < 0.5:
            y = x
        x, y = (4096, *x), (4096 + 2 * rng.randint(-60, 60), *y)
        want = bool(covered(shape, x, kx) & covered(shape, y, ky))
        got = ask(L, shape, x, kx, y, ky)
        if len(distances(shape, x, kx) | distances(shape, y, ky)) <= 2:
            assert got == want, (shape, x, kx, y, ky)
        else:
            assert got or not want, (shape, x, kx, y, ky)        # (may be turned down without need)
        seen[int(want)] += 1
    assert min(seen.values()) > 1000


def test_long_ones(L):
    """Sizes that nobody could count through: records of a gate, an input and an output side by side, one element apart or shared."""
    shape = (1000, 1 << 20, 64)
    for step in (192, 1 << 20):
        for batch in (step << 20, (step << 20) + 7):
            for k, (first, second) in enumerate([(0, 64), (0, 63), (64, 128), (65, 128), (128, 64), (127, 64)]):
                x, y = (4096 + 4 * first, batch, step), (4096 + 4 * second, batch, step)
                assert ask(L, shape, x, F32, y, F32) == k % 2, (step, batch, first, second)
            far = (4096 + 4 * (999 * batch + ((1 << 20) - 1) * step + 63), batch, step)
            assert ask(L, shape, (4096, batch, step), F32, far, F32) == 1
            assert ask(L, shape, (4096, batch, step), F32, (far[0] + 4, batch, step), F32) == 0
    assert ask(L, (1, 0, 64), (4096, 0, 64), F32, (4096, 0, 64), F32) == 0          # no steps: nothing is read or written


def forward(L, a, b, h, h0=None, reset=None, last=None, shape=(2, 10, 8)):
    r = [ctypes.byref(binding._Sequence(*q)) for q in (a, b, h)]
    return L.rls_linear_scan(ctypes.byref(binding._ScanShape(*shape, F32, F32, 0)), r[0], r[1], h0, reset, r[2], last, None, 0, None)


def backward(L, a, h, dh, da, db, h0=None, reset=None, dlast=None, dh0=None, shape=(2, 10, 8)):
    r = [ctypes.byref(binding._Sequence(*q)) for q in (a, h, dh, da, db)]
    return L.rls_linear_scan_backward(ctypes.byref(binding._ScanShape(*shape, F32, F32, 0)), r[0], r[1], r[2], h0, reset, dlast, r[3], r[4], dh0, None, 0, None)


def test_calls_turn_them_down(L):
    """Addresses are made up: every call here is turned down before anything is enqueued."""
    at = lambda k: (4096 + 65536 * k, 80, 8)             # noqa: E731
    place = lambda k: ctypes.c_void_p(4096 + 65536 * k)  # noqa: E731
    shifted = lambda k: (4096 + 65536 * k + 16, 80, 8)   # noqa: E731
    for h in (at(0), at(1), shifted(0), shifted(1)):
        assert forward(L, at(0), at(1), h) == SHAPE
    assert forward(L, at(0), at(1), at(2), h0=place(2)) == SHAPE
    assert forward(L, at(0), at(1), at(2), reset=place(2)) == SHAPE
    for k in (0, 1, 2):
        assert forward(L, at(0), at(1), at(2), last=place(k)) == SHAPE
    assert forward(L, at(0), at(1), at(2), reset=place(3), last=place(3)) == SHAPE
    assert forward(L, at(0), at(1), at(2), h0=place(3), last=ctypes.c_void_p(4096 + 65536 * 3 + 4)) == SHAPE
    for k in (0, 1, 2):
        assert backward(L, at(0), at(1), at(2), at(k), at(4)) == backward(L, at(0), at(1), at(2), at(3), at(k)) == SHAPE
        assert backward(L, at(0), at(1), at(2), at(3), at(4), dh0=place(k)) == SHAPE
    assert backward(L, at(0), at(1), at(2), at(3), at(3)) == backward(L, at(0), at(1), at(2), at(3), shifted(3)) == SHAPE
    for k in (3, 4):
        assert backward(L, at(0), at(1), at(2), at(3), at(4), h0=place(k)) == SHAPE
        assert backward(L, at(0), at(1), at(2), at(3), at(4), dlast=place(k)) == SHAPE
        assert backward(L, at(0), at(1), at(2), at(3), at(4), reset=place(k)) == SHAPE
        assert backward(L, at(0), at(1), at(2), at(3), at(4), dh0=place(k)) == SHAPE
    assert backward(L, at(0), at(1), at(2), at(3), at(4), dlast=place(5), dh0=ctypes.c_void_p(4096 + 65536 * 5 + 8)) == SHAPE
    assert backward(L, at(0), at(1), at(2), at(3), at(4), h0=place(5), dh0=place(5)) == SHAPE
