"""What rls_gated_delta turns down before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1905_12799_amd import binding

INVALID, NULL, SHAPE, WORKSPACE = -1, -2, -3, -4
BASE = 1 << 24
NAMES = ("q", "k", "v", "o", "dq", "dk", "dv", "g", "beta", "state", "reset", "last", "dlast", "dg", "dbeta", "dstate", "ws")
AT = {name: BASE * (i + 1) for i, name in enumerate(NAMES)}            # never dereferenced: a check fails first
B, T, H, HK, K, V = 2, 100, 4, 2, 16, 24


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def shape(batch=B, steps=T, heads=H, key_heads=HK, key_dim=K, value_dim=V, type=0):
    return binding._DeltaShape(batch, steps, heads, key_heads, key_dim, value_dim, type, 1.0)


def view(name, heads, dim, at=None, batch=None, step=None, head=None):
    return binding._Heads(AT[name] if at is None else at, T * heads * dim if batch is None else batch, heads * dim if step is None else step, dim if head is None else head)


def need(L, backward, **o):
    return L.rls_gated_delta_workspace_bytes(ctypes.byref(shape(**o)), backward)


def forward(L, sizes=None, bytes=0, **o):
    a = {**AT, **{n: x for n, x in o.items() if not isinstance(x, binding._Heads)}}
    h = {n: o[n] if isinstance(o.get(n), binding._Heads) else view(n, HK if n in "qk" else H, K if n in "qk" else V, a[n]) for n in ("q", "k", "v", "o")}
    r = {n: ctypes.byref(x) for n, x in h.items()}
    return L.rls_gated_delta(ctypes.byref(shape(**(sizes or {}))), r["q"], r["k"], r["v"], a["g"], a["beta"], a["state"], a["reset"], r["o"], a["last"], a["ws"], bytes, None)


def backward(L, sizes=None, bytes=0, **o):
    a = {**AT, **{n: x for n, x in o.items() if not isinstance(x, binding._Heads)}}
    h = {n: o[n] if isinstance(o.get(n), binding._Heads) else view(n, HK if n.endswith(("q", "k")) else H, K if n.endswith(("q", "k")) else V, a[n])
         for n in ("q", "k", "v", "o", "dq", "dk", "dv")}
    r = {n: ctypes.byref(x) for n, x in h.items()}
    return L.rls_gated_delta_backward(ctypes.byref(shape(**(sizes or {}))), r["q"], r["k"], r["v"], a["g"], a["beta"], a["state"], a["reset"], r["o"], a["dlast"], r["dq"],
                                      r["dk"], r["dv"], a["dg"], a["dbeta"], a["dstate"], a["ws"], bytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_sizes(L, call):
    for bad in (dict(batch=0), dict(steps=-1), dict(heads=0), dict(key_heads=0), dict(key_dim=0), dict(key_dim=129), dict(value_dim=0), dict(value_dim=513), dict(type=3),
                dict(type=-1), dict(batch=1 << 18), dict(batch=1 << 16, heads=4), dict(steps=(1 << 26) + 1), dict(batch=1 << 10, steps=1 << 24, heads=2), dict(batch=1 << 40)):
        assert call(L, bad) == INVALID, bad
        assert need(L, 0, **bad) == need(L, 1, **bad) == INVALID
    assert call(L, dict(key_heads=3)) == SHAPE
    assert L.rls_gated_delta(None, *[None] * 10, 0, None) == NULL
    assert L.rls_gated_delta_workspace_bytes(None, 0) == NULL


def test_pointers(L):
    for name in ("q", "k", "v", "o", "g", "beta"):
        assert forward(L, **{name: 0}) == NULL, name
    for name in ("q", "k", "v", "o", "dq", "dk", "dv", "g", "beta", "dg", "dbeta"):
        assert backward(L, **{name: 0}) == NULL, name


def test_strides(L):
    # what is written may not overlap itself, what is read may not run backwards or further than memory reaches
    for bad in (view("o", H, V, step=H * V - 1), view("o", H, V, head=V - 1), view("o", H, V, batch=0), view("o", H, V, head=0)):
        assert forward(L, o=bad) == SHAPE
    for name in ("dq", "dk", "dv"):
        heads, dim = (HK, K) if name != "dv" else (H, V)
        assert backward(L, **{name: view(name, heads, dim, step=heads * dim - 1)}) == SHAPE
    for bad in (view("q", HK, K, step=-1), view("q", HK, K, batch=1 << 41), view("q", HK, K, step=1 << 38)):
        assert forward(L, q=bad) == SHAPE


def test_workspace_and_overlaps(L):
    for backward_pass, call in ((0, forward), (1, backward)):
        n = need(L, backward_pass)
        assert n > 0 and n % 256 == 0
        assert call(L, ws=None, bytes=n) == call(L, bytes=n - 1) == call(L, ws=AT["ws"] + 128, bytes=n) == WORKSPACE
        assert call(L, bytes=n, ws=AT["state"]) == SHAPE
    n = need(L, 0)
    for name, where in (("last", "q"), ("last", "reset"), ("last", "g"), ("last", "o"), ("o", "v"), ("o", "state")):
        assert forward(L, bytes=n, **{name: AT[where]}) == SHAPE, (name, where)
    assert forward(L, bytes=n, last=AT["state"] + 4) == SHAPE
    n = need(L, 1)
    for name, where in (("dstate", "state"), ("dq", "q"), ("dk", "dq"), ("dg", "g"), ("dbeta", "dlast"), ("dv", "dg")):
        assert backward(L, bytes=n, **{name: AT[where]}) == SHAPE, (name, where)
    assert backward(L, bytes=n, dstate=AT["dlast"] + 4) == SHAPE
    assert need(L, 0, steps=1) == need(L, 0, steps=0) == need(L, 1, steps=0) == 0 < need(L, 1, steps=1)
    # long sequences of many heads are cut: the workspace stays bounded
    assert need(L, 0, batch=1, steps=1 << 26, heads=32, key_dim=128, value_dim=128) < 1 << 30
    assert need(L, 1, batch=1, steps=1 << 20, heads=32, key_dim=128, value_dim=128) < 5 << 30


def test_binding_looks_at_its_arguments():
    q, v, g = torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 2)
    for bad in (lambda: binding.gated_delta(q, q, v, g, g), lambda: binding.gated_delta(q[0], q[0], v, g, g), lambda: binding.gated_delta(q, q[:, :, :1], v, g, g),
                lambda: binding.gated_delta(q.double(), q.double(), v.double(), g, g), lambda: binding.gated_delta_backward(q, q, v, g, g, v)):
        with pytest.raises((ValueError, RuntimeError)):
            bad()
