"""What rls_token_logprobs and rls_distill_loss turn down before anything is enqueued (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_1905_12799_amd import binding

INVALID, NULL, SHAPE, WORKSPACE = -1, -2, -3, -4
BASE = 1 << 20
P = {name: BASE * (i + 1) for i, name in enumerate(("logits", "token", "temperature", "logprob", "entropy", "best", "best_token", "norm", "ws", "dlogprob", "dentropy",
                                                    "dlogits", "teacher"))}            # never dereferenced: a check fails first


@pytest.fixture(scope="module")
def L():
    return binding.lib()


def forward(L, **o):
    a = {**P, "type": 0, "rows": 4, "n": 10, "ld": 10, "top": 2, "bytes": 0, **o}
    return L.rls_token_logprobs(a["logits"], a["type"], a["rows"], a["n"], a["ld"], a["token"], a["temperature"], a["top"], a["logprob"], a["entropy"], a["best"],
                                a["best_token"], a["norm"], a["ws"], a["bytes"], None)


def backward(L, **o):
    a = {**P, "type": 0, "rows": 4, "n": 10, "ld": 10, "ldd": 10, **o}
    return L.rls_token_logprobs_backward(a["logits"], a["type"], a["rows"], a["n"], a["ld"], a["token"], a["temperature"], a["norm"], a["entropy"], a["dlogprob"],
                                         a["dentropy"], a["dlogits"], a["ldd"], None)


def distill(L, **o):
    a = {**P, "type": 0, "rows": 4, "n": 10, "ld": 10, "k": 3, "kind": 0, "bytes": 0, **o}
    return L.rls_distill_loss(a["logits"], a["type"], a["rows"], a["n"], a["ld"], a["token"], a["teacher"], a["kind"], a["k"], a["temperature"], a["logprob"], a["norm"],
                              a["ws"], a["bytes"], None)


def distill_backward(L, **o):
    a = {**P, "type": 0, "rows": 4, "n": 10, "ld": 10, "ldd": 10, "k": 3, "kind": 0, **o}
    return L.rls_distill_loss_backward(a["logits"], a["type"], a["rows"], a["n"], a["ld"], a["token"], a["teacher"], a["kind"], a["k"], a["temperature"], a["norm"],
                                       a["dlogprob"], a["dlogits"], a["ldd"], None)


@pytest.mark.parametrize("call", [forward, backward, distill, distill_backward])
def test_sizes(L, call):
    assert call(L, rows=0) == call(L, rows=-1) == call(L, rows=(1 << 26) + 1) == INVALID
    assert call(L, n=0) == call(L, n=(1 << 24) + 1, ld=1 << 25) == INVALID
    assert call(L, type=3) == call(L, type=-1) == INVALID
    assert call(L, ld=9) == SHAPE
    assert call(L, logits=0) == NULL


def test_forward(L):
    assert forward(L, top=-1) == forward(L, top=129) == INVALID
    assert forward(L, token=0) == forward(L, logprob=0) == forward(L, best=0) == forward(L, best_token=0) == NULL
    for a, b in (("logprob", "logits"), ("entropy", "token"), ("best", "norm"), ("norm", "temperature"), ("best_token", "best")):
        assert forward(L, **{a: P[b]}) == SHAPE
    assert forward(L, logprob=P["logits"] + 4 * 39) == SHAPE                      # the last logit
    need = L.rls_token_logprobs_workspace_bytes(4, 100000, 2)
    assert need > 0
    big = dict(n=100000, ld=100000, logits=1 << 40)
    assert forward(L, **big, ws=0, bytes=need) == forward(L, **big, bytes=need - 1) == forward(L, **big, ws=P["ws"] + 64, bytes=need) == WORKSPACE
    assert forward(L, **{**big, "ws": big["logits"]}, bytes=need) == SHAPE
    assert L.rls_token_logprobs_workspace_bytes(0, 1, 0) == L.rls_token_logprobs_workspace_bytes(1, 0, 0) == L.rls_token_logprobs_workspace_bytes(1, 1, 129) == INVALID
    assert L.rls_token_logprobs_workspace_bytes(1 << 26, 1 << 24, 128) == 0
    for rows in (1, 3, 100, 511):
        for top in (0, 1, 128):
            assert 0 < L.rls_token_logprobs_workspace_bytes(rows, 1 << 24, top) < 1 << 26


def test_backward(L):
    assert backward(L, norm=0) == backward(L, token=0) == backward(L, entropy=0) == backward(L, dlogits=0) == NULL
    assert backward(L, ldd=9) == SHAPE
    for bad in (dict(dlogits=P["logits"] + 4), dict(dlogits=P["logits"], ldd=11), dict(dlogits=P["norm"]), dict(dlogits=P["dentropy"] - 4 * 39)):
        assert backward(L, **bad) == SHAPE, bad


def test_distill(L):
    for call in (distill, distill_backward):
        assert call(L, token=0) == call(L, teacher=0) == NULL
        assert call(L, k=0) == call(L, k=129) == call(L, kind=3) == INVALID
    assert distill(L, logprob=0) == distill_backward(L, norm=0) == distill_backward(L, dlogprob=0) == distill_backward(L, dlogits=0) == NULL
    assert distill(L, norm=P["teacher"] + 8) == distill(L, logprob=P["token"]) == SHAPE
    assert distill_backward(L, dlogits=P["teacher"]) == distill_backward(L, dlogits=P["logits"] - 4) == SHAPE
    need = L.rls_distill_loss_workspace_bytes(4, 100000)
    assert need > 0 and distill(L, n=100000, ld=100000, logits=1 << 40, bytes=need - 1) == WORKSPACE


def test_binding_looks_at_its_arguments():
    x = torch.zeros(4, 10)
    k = torch.zeros(4, dtype=torch.int32)
    for bad in (lambda: binding.token_logprobs(x, k), lambda: binding.distill_loss(x, k[:, None], x[:, :1]),
                lambda: binding.token_logprobs_backward(x, k, x[:, :2], None, k.float()), lambda: binding.distill_loss_backward(x, k[:, None], x[:, :1], x[:, :2], k.float())):
        with pytest.raises(ValueError):
            bad()
    assert binding.MAX_TOP == 128 and binding.LogProbs._fields == ("logprob", "entropy", "top_logprob", "top_token", "norm")
    assert ctypes.sizeof(ctypes.c_void_p) == 8
