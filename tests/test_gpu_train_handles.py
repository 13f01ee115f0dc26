"""The training handles on the GPU: tensors that change their memory."""
import pytest
import torch

from paper_2609_28053_amd import AdamW
from test_gpu_balance import say

pytestmark = pytest.mark.gpu

D = dict(device="cuda")


def tensors(seed, *shapes):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(s, generator=g, **D) for s in shapes]


SHAPES = ((64, 33), (5,), (300,))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_parameter_that_moves_is_followed(bits):
    """p.data = ... between two steps: the new memory gets the step, bit for bit, and the old one keeps its values."""
    say(f"adamw {bits} bits, a parameter moves")
    still, moved = tensors(0, *SHAPES), tensors(0, *SHAPES)
    a, b = AdamW(still, lr=1e-2, state_bits=bits), AdamW(moved, lr=1e-2, state_bits=bits)
    first, second = tensors(1, *SHAPES), tensors(2, *SHAPES)
    a.step(first)
    b.step(first)
    old = moved[0].data
    was = old.clone()
    moved[0].data = old.clone()
    a.step(second)
    b.step(second)
    assert all(torch.equal(p, q) for p, q in zip(still, moved))
    assert torch.equal(old, was) and not torch.equal(moved[0], was)
