"""What GatedExperts refuses, and that a refused call leaves it as it was."""
import pytest
import torch

from paper_2609_28053_amd import ExpertRows, GatedExperts
from test_gpu_balance import say

pytestmark = pytest.mark.gpu
D = dict(device="cuda")


def made(T=50, E=8, K=2, H=72, F=40):
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s: torch.randn(s, generator=g, **D).to(torch.bfloat16)  # noqa: E731
    up, down, x = new(E, 2 * F, H), new(E, H, F), new(T, H)
    rows = ExpertRows(T, E, K)
    rows.plan(torch.stack([torch.randperm(E, generator=g, **D)[:K] for _ in range(T)]).to(torch.int32))
    return up, down, x, rows, GatedExperts(up, down)


def test_refresh_takes_both_weights_or_none():
    say("refresh takes both or none")
    up, down, x, rows, experts = made()
    want, _ = experts.forward(x, rows)
    other = -2 * up
    for bad in (down[:4], down[:, :, :32], down.double(), down.cpu(), down.transpose(1, 2).contiguous().transpose(1, 2), None):
        with pytest.raises((ValueError, TypeError, AttributeError)):
            experts.refresh(other, bad)
        with pytest.raises((ValueError, TypeError, AttributeError)):
            experts.refresh(bad, down)
        got, _ = experts.forward(x, rows)
        assert torch.equal(got, want)
    experts.refresh(other, down)
    got, _ = experts.forward(x, rows)
    assert not torch.equal(got, want)


def test_rows_of_another_width_are_refused():
    """Rows of 72 and of 80 elements have codes of the same width, 128."""
    say("rows of another width")
    up, down, x, rows, experts = made()
    wide = torch.zeros((50, 80), dtype=torch.bfloat16, **D)
    for train in (False, True):
        with pytest.raises(ValueError, match="80"):
            experts.forward(wide, rows, train=train)
    out, saved = experts.forward(x, rows)
    with pytest.raises(ValueError, match="80"):
        experts.backward(torch.zeros((100, 80), dtype=torch.bfloat16, **D), saved)
    experts.backward(torch.zeros_like(out), saved)
