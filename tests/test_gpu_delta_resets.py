"""rls.gated_delta: what lies behind a reset, or a gate that keeps nothing, does not reach what lies before it, and the other way round.

Tolerances as in test_gpu_delta: errors of a sequence by itself, relative to its own largest value."""
import pytest
import torch

from tests.test_gpu_delta import close, gradients, inputs, rls              # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T,cut", [(64, 63), (60, 7), (100, 40), (200, 128), (200, 150)])
def test_gradients_before_a_cut_beside_large_ones_behind_it(rls, T, cut, kind):     # noqa: F811
    """Gradients behind the cut 2^20 times as large: those by the gates before it keep their digits."""
    shape = B, _, H, HK, K, V = 2, T, 4, 2, 48, 40
    for gate in (False, True):
        d = inputs(*shape, kind, T + cut)
        if gate:
            d["g"][:, cut] = -torch.inf
        else:
            d["reset"] = torch.zeros(B, T, dtype=torch.uint8, device="cuda")
            d["reset"][:, cut] = 1
        do = torch.randn(B, T, H, V, generator=torch.Generator().manual_seed(cut)).cuda()
        do[:, cut:] *= 2.0 ** 20 if kind == "f32" else 2.0 ** 12
        do = do.to(d["v"].dtype)
        names = ("q", "k", "v", "g", "beta")
        got = dict(zip(names + ("state",), rls.gated_delta_backward(*(d[n] for n in names), do, d["state"], d["reset"], scale=0.3)))
        alone = {n: (None if d[n] is None else d[n] if n == "state" else d[n][:, :cut].contiguous()) for n in names + ("state", "reset")}
        want = gradients(alone, do[:, :cut], None, 0.3)
        terms = (alone["beta"] * want["beta"]).abs().max()
        for n, w in want.items():
            close(got[n] if n == "state" else got[n][:, :cut], w, T, K, 2, (n, gate), terms if n == "g" else 0.0)
