"""What rls_sample, rls_linear_scan and rls_adamw_step turn down before anything is enqueued (no GPU needed)."""
import ctypes

import pytest

from paper_1905_12799_amd import binding

INVALID, NULL, SHAPE, WORKSPACE = -1, -2, -3, -4
FAKE, NONE = ctypes.c_void_p(4096), ctypes.c_void_p(None)        # never dereferenced: a check fails first


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def sample(L, logits=FAKE, type=0, rows=4, n=10, ld=10, uniform=FAKE, token=FAKE):
    return L.rls_sample(logits, type, rows, n, ld, uniform, None, None, None, None, token, None, None, 0, None)


def test_sample(L):
    assert sample(L, logits=NONE) == sample(L, uniform=NONE) == sample(L, token=NONE) == NULL
    assert sample(L, rows=0) == sample(L, rows=-1) == sample(L, rows=(1 << 26) + 1) == INVALID
    assert sample(L, n=0) == sample(L, n=-3) == sample(L, n=(1 << 24) + 1, ld=1 << 25) == INVALID
    assert sample(L, type=3) == sample(L, type=-1) == INVALID
    assert sample(L, ld=9) == SHAPE
    assert L.rls_sample_workspace_bytes(0, 5) == L.rls_sample_workspace_bytes(5, 0) == INVALID
    assert L.rls_sample_workspace_bytes(1 << 26, 1 << 24) >= 0
    # a shape that needs a workspace is turned down without one, with one that is too small, and with one that is not aligned
    for rows, n in ((1, 1 << 24), (1, 8388608)):
        need = L.rls_sample_workspace_bytes(rows, n)
        if need > 0:
            call = lambda ws, b: L.rls_sample(FAKE, 0, rows, n, n, FAKE, None, None, None, None, FAKE, None, ws, b, None)      # noqa: E731
            assert call(NONE, need) == call(FAKE, need - 1) == call(ctypes.c_void_p(4096 + 64), need) == WORKSPACE


def seq(data=4096, batch=1000, step=10):
    return binding._Sequence(data, batch, step)


def scan(L, shape=(2, 100, 10, 0, 0, 0), a=None, b=None, h=None):
    a, b, h = a or seq(), b or seq(), h or seq()
    return L.rls_linear_scan(ctypes.byref(binding._ScanShape(*shape)), ctypes.byref(a), ctypes.byref(b), None, None, ctypes.byref(h), None, None, 0, None)


def backward(L, shape=(2, 100, 10, 0, 0, 0), **other):
    q = {k: other.get(k) or seq() for k in ("a", "h", "dh", "da", "db")}
    r = {k: ctypes.byref(v) for k, v in q.items()}
    return L.rls_linear_scan_backward(ctypes.byref(binding._ScanShape(*shape)), r["a"], r["h"], r["dh"], None, None, None, r["da"], r["db"], None, None, 0, None)


def test_linear_scan(L):
    assert L.rls_linear_scan(None, None, None, None, None, None, None, None, 0, None) == NULL
    assert L.rls_linear_scan(ctypes.byref(binding._ScanShape(1, 1, 1, 0, 0, 0)), None, None, None, None, None, None, None, 0, None) == NULL
    for call in (scan, backward):
        for shape in ((0, 100, 10, 0, 0, 0), (2, -1, 10, 0, 0, 0), (2, 100, 0, 0, 0, 0), (2, (1 << 26) + 1, 10, 0, 0, 0), (1 << 20, 100, 1 << 20, 0, 0, 0),
                      (2, 100, 10, 3, 0, 0), (2, 100, 10, 0, 1, 0), (2, 100, 10, 1, 2, 0), (2, 100, 10, -1, 0, 0)):
            assert call(L, shape) == INVALID, shape
        assert call(L, a=seq(data=None)) == NULL
        assert call(L, a=seq(batch=-1)) == call(L, a=seq(step=-10)) == SHAPE
    # what is written may not overlap itself
    for bad in (seq(step=9), seq(step=0), seq(batch=999), seq(batch=0), seq(batch=5, step=20)):
        assert scan(L, h=bad) == SHAPE and backward(L, da=bad) == SHAPE and backward(L, db=bad) == SHAPE
    assert L.rls_linear_scan_workspace_bytes(0, 1, 1) == L.rls_linear_scan_workspace_bytes(1, -1, 1) == INVALID
    assert L.rls_linear_scan_workspace_bytes(1, 0, 1) >= 0
    need = L.rls_linear_scan_workspace_bytes(1, 1 << 20, 64)
    if need > 0:
        call = lambda ws, b: L.rls_linear_scan(ctypes.byref(binding._ScanShape(1, 1 << 20, 64, 0, 0, 0)), ctypes.byref(seq(step=64, batch=1 << 26)),      # noqa: E731
                                               ctypes.byref(seq(step=64, batch=1 << 26)), None, None, ctypes.byref(seq(step=64, batch=1 << 26)), None, ws, b, None)
        assert call(NONE, need) == call(FAKE, need - 1) == call(ctypes.c_void_p(4096 + 128), need) == WORKSPACE


def adamw(L, tensors, step=1, bits=32, beta1=0.9, beta2=0.999, eps=1e-8, lr=1e-3, decay=0.0, n=None):
    arr = (binding._AdamwTensor * max(1, len(tensors)))(*tensors)
    o = binding._AdamwOptions(lr, beta1, beta2, eps, decay, step, 0, bits, None)
    return L.rls_adamw_step(arr, len(tensors) if n is None else n, ctypes.byref(o), None)


def tensor(n=10, p=0, g=0, param=4096, grad=4096, master=None, m=4096, v=4096, ms=None, vs=None):
    return binding._AdamwTensor(n, p, g, param, grad, master, m, v, ms, vs)


def test_adamw(L):
    assert L.rls_adamw_step(None, 0, None, None) == NULL
    assert L.rls_adamw_step(None, 1, ctypes.byref(binding._AdamwOptions(1e-3, 0.9, 0.999, 1e-8, 0.0, 1, 0, 32, None)), None) == NULL
    nan = float("nan")
    for bad in ({"step": 0}, {"bits": 16}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": nan}, {"eps": -1.0}, {"eps": nan}, {"lr": nan},
                {"lr": float("inf")}, {"decay": nan}, {"n": -1}):
        assert adamw(L, [tensor()], **bad) == INVALID, bad
    for bad in (tensor(n=-1), tensor(n=1 << 40), tensor(p=3), tensor(p=0, g=1), tensor(p=1, g=2), tensor(master=4096)):
        assert adamw(L, [bad]) == INVALID
    for bad in (tensor(param=None), tensor(grad=None), tensor(m=None), tensor(v=None)):
        assert adamw(L, [bad]) == NULL
    assert adamw(L, [tensor()], bits=8) == adamw(L, [tensor(ms=4096)], bits=8) == NULL
    # nothing to do: nothing is enqueued
    assert adamw(L, []) == 0
    assert adamw(L, [tensor(n=0, param=None, grad=None, m=None, v=None)]) == 0


def test_binding_checks_its_arguments():
    import torch
    x = torch.zeros(2, 3)
    with pytest.raises(ValueError):
        binding.sample(x, torch.zeros(2))
    with pytest.raises(ValueError):
        binding.linear_scan(torch.zeros(1, 2, 3), torch.zeros(1, 2, 3))
    with pytest.raises(ValueError):
        binding.linear_scan(torch.zeros(1, 2, 3, dtype=torch.float16), torch.zeros(1, 2, 3))
    with pytest.raises(ValueError):
        binding.AdamW([x])
    with pytest.raises(ValueError):
        binding.AdamW([], state_bits=4)
