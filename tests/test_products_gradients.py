"""The products have no backward pass: operands that require a gradient are refused (no GPU needed)."""
import pytest
import torch

from paper_2510_03293_amd import binding as B

T, H, F, E, k = 4, 64, 32, 4, 2


class Routed:
    def __init__(self):
        self.k = k
        self.permutation = torch.zeros(T * k, dtype=torch.int32)
        self.expert_offsets = torch.zeros(E + 1, dtype=torch.int32)
        self.expert_ids = torch.zeros(T, k, dtype=torch.int32)
        self.weights = torch.zeros(T, k)


def layer():
    return dict(hidden=torch.zeros(T, H), w_up=torch.zeros(E, 2 * F, H), w_down=torch.zeros(E, H, F), routed=Routed(),
                base=torch.zeros(T, H))


def projection():
    return dict(x=torch.zeros(T, H), w=torch.zeros(8, H), a_down=torch.zeros(2, 8, H), a_up=torch.zeros(2, 8, 8),
                scales=torch.ones(2), request_offsets=torch.zeros(3, dtype=torch.int32),
                request_adapters=torch.zeros(2, dtype=torch.int32))


@pytest.mark.parametrize("call,make,name", [(B.experts, layer, n) for n in ("hidden", "w_up", "w_down", "base", "weights")]
                         + [(B.project_adapted, projection, n) for n in ("x", "w", "a_down", "a_up", "scales")])
def test_operands_that_require_a_gradient(call, make, name):
    given = make()
    (given["routed"].weights if name == "weights" else given[name]).requires_grad_()
    with pytest.raises(ValueError, match=f"{name} requires a gradient"):
        call(**given)
    # without gradients the call goes on to its other checks: these tensors are not on a GPU
    with torch.no_grad(), pytest.raises(ValueError, match="current GPU"):
        call(**given)
    with pytest.raises(ValueError, match="current GPU"):
        call(**make())
