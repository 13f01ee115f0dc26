"""The router backward inside the balance loss's gradient against the router backward alone."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_balance_loss import Case, check, cuda, run

pytestmark = pytest.mark.gpu


def spread(c, seed):
    """Logits of every size: to 30, to 90 and past 100 of both signs, and masked ones, most rows of one kind."""
    x = c.z.to(torch.float32)
    rng = np.random.default_rng(seed)
    x[::3] *= 12.0
    x[1::5] *= 30.0
    x[7::11] = torch.from_numpy(rng.choice([-200.0, -104.0, -95.0, -88.0, -87.5, -64.0, -32.0, 0.0, 31.75, 32.0, 63.5, 64.0,
                                            87.5, 95.0, 103.0, 150.0], size=x[7::11].shape).astype(np.float32))
    x[3::13, ::2] = -float("inf")
    c.z = x.to(torch.bfloat16)
    c.x = c.z.to(torch.float64).numpy()
    fin = np.abs(c.x[np.isfinite(c.x)])
    c.eps = (2 * fin.max() + 24) * 2.0 ** -23


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("E,K", [(8, 1), (8, 5), (16, 3), (32, 4), (64, 6), (128, 40), (256, 8)])
def test_the_same_bits_without_the_loss(eqb, E, K, softmax):  # noqa: F811
    """With alpha = 0 every gradient of a finite logit is (g + inj) sigmoid'(z), bit for bit eqb_lei_router_backward's,
    whatever the logit's size; subnormal ones are there in both."""
    c = Case(E + K, 1500, E, K, 3)
    spread(c, E)
    say(f"fused backward, E={E} K={K} softmax={softmax}")
    got = run(eqb, c, softmax, alpha=0.0)["gz"]
    gz = torch.empty((c.T, c.E), device="cuda")
    eqb.eqb_lei_router_backward(c.z.view(torch.int16).cuda(), cuda(c.idx), cuda(c.gs), gz, cuda(c.inj), c.part)
    want = gz.cpu().numpy()
    assert np.array_equal(got, want)
    assert np.any((np.abs(want) > 0) & (np.abs(c.x) > 90))


@pytest.mark.parametrize("E,K", [(8, 2), (64, 6), (256, 8)])
def test_large_logits_against_the_oracle(eqb, E, K):  # noqa: F811
    """The whole gradient, loss and router, at the tolerance of the balance loss."""
    c = Case(E, 900, E, K, 2, mask=True)
    spread(c, E + 1)
    say(f"fused backward against the oracle, E={E}")
    check(c, run(eqb, c, False), False)
    p = O.probabilities(c.x, False)
    assert np.all(np.isfinite(p))


@pytest.mark.parametrize("router", [False, True])
@pytest.mark.parametrize("softmax", [False, True])
def test_a_logit_that_is_no_number_spoils_its_row(eqb, softmax, router):  # noqa: F811
    """NaN in a valid token's logits: its whole row of the gradient is NaN, the other rows keep their bits (the loads,
    tokens and losses of the gradient are given)."""
    c = Case(31, 200, 64, 4, 2)
    say(f"a NaN logit, softmax={softmax} router={router}")
    load, tokens = cuda(np.full((2, 64), 3, dtype=np.int32)), cuda(np.full(2, 100, dtype=np.int32))
    kw = dict(topk_idx=cuda(c.idx), grad_score=cuda(c.gs), inj=cuda(c.inj)) if router else {}
    out = []
    for bad in (False, True):
        x = c.z.clone()
        if bad:
            x[17, 5] = x[150, 63] = float("nan")
        gz = torch.empty((200, 64), device="cuda")
        eqb.eqb_balance_backward(x.view(torch.int16).cuda(), load, tokens, 4, 0.3, cuda(c.gl), gz, part_off=c.part,
                                 score=eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID, **kw)
        out.append(gz.cpu().numpy())
    spoilt = np.zeros(200, dtype=bool)
    spoilt[[17, 150]] = True
    assert np.isnan(out[1][spoilt]).all() and np.array_equal(out[0][~spoilt], out[1][~spoilt])
