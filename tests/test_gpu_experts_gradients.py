"""The whole backward pass of GatedExperts, and of the layer around it, against the gradients of the same layer without
codes in binary64, written from the formulas: no call of the library makes a reference here.

Tolerance.  A code is within 2^-4 of its value or, below the normal codes, within 2^-10 of its block's scale, which is less
than top / 224: 2^-17 of the largest value.  Inputs and weights are codes themselves, so that the gate is right to binary32.  A
gradient of the rows goes through the codes of grad_out and through those of the gate's gradient, the weights' gradients through
one code of each factor but for x and up; errors of factors are multiplied out.  All sums and roundings of binary32: 2^-15 of
the magnitudes, for sums of up to 513 terms."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from paper_2609_28053_amd import ExpertRows, GatedExperts, ScoredRouter
from test_gpu_balance import say

pytestmark = pytest.mark.gpu
SUMS = 2.0 ** -15


def off_by(v):
    """How far the codes of v may be off."""
    return 2.0 ** -4 * np.abs(v) + 2.0 ** -17 * np.abs(v).max()


@pytest.mark.parametrize("T,E,K,H,F", [(1, 8, 1, 8, 4), (40, 8, 2, 8, 4), (300, 16, 3, 150, 70), (513, 8, 2, 130, 129)])
def test_all_gradients(T, E, K, H, F):
    say(f"all gradients T={T} E={E} K={K} H={H} F={F}")
    rng = np.random.default_rng(T + H)
    x = rng.integers(-4, 5, size=(T, H)) * 0.25
    up, down = rng.integers(-3, 4, size=(E, 2 * F, H)) * 2.0 ** -4, rng.integers(-3, 4, size=(E, H, F)) * 2.0 ** -4
    z, gy = rng.normal(size=(T, E)).astype(np.float32).astype(np.float64), rng.normal(size=(T, H)).astype(np.float32).astype(np.float64)
    t = lambda v: torch.from_numpy(np.ascontiguousarray(v)).to(torch.float32).cuda()  # noqa: E731
    router, rows, experts = ScoredRouter(E, K), ExpertRows(T, E, K), GatedExperts(t(up), t(down))
    idx, weight = router.forward(t(z))
    rows.plan(idx)
    out, saved = experts.forward(t(x), rows)
    grad_out, _ = rows.combine_backward(t(gy), out, weight)
    grad_rows, grad_up, grad_down = experts.backward(grad_out, saved)
    grad_x = rows.combine(grad_rows)

    ii = np.argsort(-z, axis=1, kind="stable")[:, :K]
    assert np.array_equal(ii, idx.cpu().numpy())
    s = 1 / (1 + np.exp(-np.take_along_axis(z, ii, 1)))
    w = s / s.sum(1, keepdims=True)
    want = [np.zeros((E, 2 * F, H)), np.zeros((E, H, F)), np.zeros((T, H))]
    tol = [np.zeros_like(v) for v in want]
    # per expert, so that the largest values are those that share its blocks
    for e in range(E):
        at = [(tt, k) for tt in range(T) for k in range(K) if ii[tt, k] == e]
        if not at:
            continue
        tok = np.array([a for a, _ in at])
        xe, ge = x[tok], gy[tok] * np.array([w[a] for a in at])[:, None]
        gate, u = np.split(xe @ up[e].T, 2, axis=1)
        sg = 1 / (1 + np.exp(-gate))
        h = gate * sg * u
        gh, dg, du = ge @ down[e], u * sg * (1 + gate * (1 - sg)), gate * sg
        size = np.abs(ge) @ np.abs(down[e])
        err = off_by(ge) @ np.abs(down[e]) + SUMS * size
        gg = np.concatenate([gh * dg, gh * du], axis=1)
        err = np.concatenate([err * np.abs(dg), err * np.abs(du)], axis=1) + 2.0 ** -20 * np.abs(gg)
        err += off_by(np.abs(gg) + err)
        want[0][e], tol[0][e] = gg.T @ xe, err.T @ np.abs(xe) + SUMS * (np.abs(gg) + err).T @ np.abs(xe)
        most = (np.abs(ge) * (1 + SUMS) + off_by(ge)).T @ (np.abs(h) * (1 + SUMS) + off_by(h))
        want[1][e], tol[1][e] = ge.T @ h, most * (1 + SUMS) - np.abs(ge).T @ np.abs(h)
        np.add.at(want[2], tok, gg @ up[e])
        np.add.at(tol[2], tok, err @ np.abs(up[e]) + SUMS * (np.abs(gg) + err) @ np.abs(up[e]))
    for name, got, v, most in zip(("up", "down", "x"), (grad_up, grad_down, grad_x), want, tol):
        off = np.abs(got.to(torch.float64).cpu().numpy() - v)
        assert (off <= most + 1e-30).all(), (name, float((off - most).max()))
        # sums of few terms tell a gradient from none; those of many are bounded by the terms' magnitudes
        assert H > 8 or (np.abs(v) > most).any()
