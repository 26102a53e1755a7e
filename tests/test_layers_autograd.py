"""The operators have their gradients as calls of their own and no history: a call whose inputs would be differentiated is refused, or their gradients
would be lost without a word.  (Nothing here gets as far as a device.)"""
import pytest
import torch

from paper_2605_29346_amd import layers

X, V = torch.zeros(4, 8), torch.zeros(8)
CALLS = {
    "linear": (lambda **t: layers.linear(t.pop("a", X), t.pop("w", X), **t), {"a": X, "w": X, "bias": V, "residual": X, "scale_a": V, "scale_w": V}),
    "linear_backward": (lambda **t: layers.linear_backward(t.pop("dy", X), t.pop("a", X), t.pop("w", X), **t), {"dy": X, "a": X, "w": X, "preact": X}),
    "dropout": (lambda **t: layers.dropout(t.pop("x", X), None, **t), {"x": X, "residual": X}),
    "rms_norm": (lambda **t: layers.rms_norm(t.pop("x", X), **t), {"x": X, "gain": V, "residual": X}),
    "rms_norm_backward": (lambda **t: layers.rms_norm_backward(t.pop("dy", X), t.pop("h", X), t.pop("rstd", V), **t), {"dy": X, "h": X, "rstd": V, "gain": V, "dh": X}),
}


@pytest.mark.parametrize("name,operand", [(name, operand) for name, (_, operands) in CALLS.items() for operand in operands])
def test_an_operand_that_wants_a_gradient_is_refused(name, operand):
    call, operands = CALLS[name]
    wants = operands[operand].clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        call(**{operand: wants})
    # what is detached, or asked for without a history, goes on to the next check
    with pytest.raises(ValueError, match="CUDA"):
        call(**{operand: wants.detach()})
    with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
        call(**{operand: wants})
