"""One balance-loss workspace over calls of other sizes, and groups whose pieces are joined in
two levels, against the binary64 oracle.

Tolerance: as for the balance loss (a probability is off by eps at most, a mean by n 2^-24
more where a lane sums n rows, a loss by that and 2^-23); every batch below is cut into at
least 128 pieces, or has less than 128 rows, so that n is T / 128 + 1 at most."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_balance_loss import Case, cuda

pytestmark = pytest.mark.gpu


def loss_of(eqb, c, ws, softmax=False, alpha=0.3):  # noqa: F811
    load = torch.full((c.P, c.E), -7, dtype=torch.int32, device="cuda")
    tokens = torch.full((c.P,), -7, dtype=torch.int32, device="cuda")
    prob, loss = torch.full((c.P, c.E), float("nan"), device="cuda"), torch.full((c.P,), float("nan"), device="cuda")
    eqb.eqb_balance_loss(c.z.view(torch.int16).cuda(), cuda(c.idx), c.K, alpha, load, tokens, prob, loss, ws,
                         cuda(c.valid, torch.bool), c.part, eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID)
    want = O.balance_loss(c.x, c.idx, c.K, alpha, c.part, c.valid, softmax)
    assert np.array_equal(load.cpu().numpy(), want[0]) and np.array_equal(tokens.cpu().numpy(), want[1])
    rel = c.eps + (c.T // 128 + 1) * 2.0 ** -24
    assert np.all(np.abs(prob.cpu().numpy() - want[2]) <= rel * want[2] + 1e-44)
    assert np.all(np.abs(loss.cpu().numpy() - want[3]) <= (rel + 2.0 ** -23) * np.abs(want[3]))
    assert not ws[:2304].any(), "both kinds of tickets are zero again"


def even(T, P):
    return [T * p // P for p in range(P + 1)]


def test_one_workspace_for_calls_of_all_sizes(eqb):  # noqa: F811
    """A buffer of the largest size serves few groups, many, few again and another E: what one call leaves in its
    scratch is no ticket of the next."""
    ws = torch.zeros(eqb.eqb_balance_workspace_size(256, 256), dtype=torch.uint8, device="cuda")
    for E, P, mask in ((256, 1, True), (256, 100, True), (256, 1, False), (64, 256, True), (256, 40, True), (8, 3, True),
                       (256, 256, False), (256, 1, True)):
        say(f"balance, one workspace, E={E} P={P} mask={mask}")
        loss_of(eqb, Case(E + P, 20000, E, 4, mask=mask, cuts=even(20000, P)), ws)


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("cuts", [[0, 30011], [0, 11, 10003, 10003, 30011], even(30011, 50)])
@pytest.mark.parametrize("E,mask", [(256, True), (256, False), (128, True)])
def test_pieces_joined_in_two_levels(eqb, softmax, cuts, E, mask):  # noqa: F811
    """More than 256 KiB of pieces (E = 256), and less (E = 128, but for 50 groups), over one, several and many groups."""
    c = Case(len(cuts) + E, 30011, E, 3, mask=mask, inf=0.01, drop=0.05, cuts=cuts)
    say(f"balance, two levels, E={E} groups={c.P} mask={mask} softmax={softmax}")
    ws = torch.zeros(eqb.eqb_balance_workspace_size(E, c.P), dtype=torch.uint8, device="cuda")
    loss_of(eqb, c, ws, softmax)


@pytest.mark.parametrize("E,T", [(256, 48 * 63 - 1), (256, 48 * 64 - 5), (256, 48 * 65), (256, 48 * 128), (256, 48 * 129 + 1),
                                 (128, 96 * 64), (8, 1536 * 64 + 11), (256, 70001)])
def test_a_lanes_sums_of_whole_lengths(eqb, E, T):  # noqa: F811
    """One block over one group, at step counts around the 64 that a lane sums before it adds to its wave's sum."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    z = (torch.randn((T, E), generator=g, device="cuda") * 1.5).to(torch.bfloat16)
    valid = torch.rand(T, generator=g, device="cuda") < 0.8
    p = torch.sigmoid(z.double())
    p = (p / p.sum(1, keepdim=True))[valid].mean(0)
    ws = torch.zeros(eqb.eqb_balance_workspace_size(E, 1), dtype=torch.uint8, device="cuda")
    load, tokens = torch.ones((1, E), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    prob, loss = torch.empty((1, E), device="cuda"), torch.empty(1, device="cuda")
    say(f"balance, one block, E={E} T={T}")
    eqb.eqb_set_max_blocks(1)
    try:
        eqb.eqb_balance_loss(z.view(torch.int16), None, 2, 1.0, load, tokens, prob, loss, ws, valid)
    finally:
        eqb.eqb_set_max_blocks(0)
    eps = (2 * float(z.float().abs().max()) + 24) * 2.0 ** -23
    assert int(tokens) == int(valid.sum())
    assert bool(((prob[0].double() - p).abs() <= (eps + 128 * 2.0 ** -24) * p).all())


def test_means_of_many_equal_rows(eqb):  # noqa: F811
    """2,000,000 copies of one row in one block: a lane adds the same number 80,000 times, so that the roundings of one
    long binary32 sum would all go one way (1e-3 and more); a lane sums 128 rows at most, and the rest is binary64."""
    E, T = 256, 2000000
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    row = torch.randn((1, E), generator=g, device="cuda").to(torch.bfloat16)
    z = row.expand(T, E).contiguous()
    p = torch.softmax(row.double(), 1)[0]
    ws = torch.zeros(eqb.eqb_balance_workspace_size(E, 1), dtype=torch.uint8, device="cuda")
    load, tokens = torch.ones((1, E), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    prob, loss = torch.empty((1, E), device="cuda"), torch.empty(1, device="cuda")
    say("balance, equal rows in one block")
    eqb.eqb_set_max_blocks(1)
    try:
        eqb.eqb_balance_loss(z.view(torch.int16), None, 2, 1.0, load, tokens, prob, loss, ws, score=eqb.EQB_SCORE_SOFTMAX)
    finally:
        eqb.eqb_set_max_blocks(0)
    eps = (2 * float(row.float().abs().max()) + 24) * 2.0 ** -23
    far = ((prob[0].double() - p).abs() / p).max()
    say(f"relative error {float(far):.1e}")
    assert float(far) <= eps + 128 * 2.0 ** -24
