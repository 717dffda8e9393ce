"""What token_logprobs and distill_loss take for a constant (no GPU needed: the calls end before anything is enqueued)."""
import pytest
import torch

from paper_1905_12799_amd import binding


@pytest.mark.parametrize("learned", [False, True])
def test_a_learned_temperature_is_turned_down(learned):
    """Without a gradient by it, it would silently not be learned."""
    x = torch.zeros(2, 5, requires_grad=learned)
    token, k = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32)
    t = torch.ones(2, requires_grad=True)
    for call in (lambda t: binding.token_logprobs(x, token, temperature=t), lambda t: binding.distill_loss(x, k, torch.zeros(2, 3), temperature=t)):
        with pytest.raises(ValueError, match="detach"):
            call(t)
        with torch.no_grad(), pytest.raises(ValueError, match="device"):       # (as far as the check of where the logits are)
            call(t)
        with pytest.raises(ValueError, match="device"):
            call(t.detach())
