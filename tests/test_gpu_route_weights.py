"""Normalized weights, and their gradient, of rows whose chosen scores are all below what binary32 holds: a bias chose
experts far below the row's largest logit (softmax), or every logit is far below zero (sigmoid).  Their ratios are
ordinary numbers.

Reference: ratios of the scores' logarithms in binary64 (log s = z - log sum exp z, or z - log(1 + exp z)).  Tolerance
(u = 2^-24): an exponential of a distance d between two chosen logits is off by d u, for the rounded distance, and 3u;
a sigmoid's other factor by 8u; a ratio has two of these, K u of the sum, its own and the scale's: r = (2 d + 22 + K + 4) u.
A gradient is such a ratio times another factor of 8u and a difference of K + 1 terms each off by 2 r: (4 r + (K + 18) u) of
the magnitudes.  2^-100 for ratios that are lost beside one of 2^-20."""
import numpy as np
import pytest
import torch

from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def want_of(z, idx, g, softmax, scale):
    """Weights [T,K], their gradient [T,E] and its magnitudes."""
    T, K = idx.shape
    w, grad, size = np.zeros((T, K)), np.zeros(z.shape), np.zeros(z.shape)
    for t in range(T):
        on = np.nonzero(idx[t] >= 0)[0]
        if not len(on):
            continue
        x = z[t, idx[t, on]]
        ls = x if softmax else x - np.logaddexp(0.0, x)
        r = np.exp(ls - ls.max())
        r /= r.sum()
        w[t, on] = scale * r
        rest = 1.0 if softmax else 1 / (1 + np.exp(x))
        np.add.at(grad[t], idx[t, on], scale * r * (g[t, on] - g[t, on] @ r) * rest)
        np.add.at(size[t], idx[t, on], abs(scale) * r * (np.abs(g[t, on]) + np.abs(g[t, on]) @ r) * rest)
    return w, grad, size


CASES = [  # E, K, groups, keep, softmax, dtype: lists of 8 and of 16, rounds (K above 16, groups below a lane's experts)
    (8, 3, 1, 1, True, "f32"), (64, 4, 1, 1, True, "bf16"), (256, 8, 8, 4, True, "bf16"), (256, 6, 8, 4, False, "bf16"),
    (128, 12, 4, 2, True, "f16"), (256, 16, 1, 1, False, "f32"), (64, 20, 1, 1, True, "f32"), (256, 7, 32, 9, False, "bf16"),
    (32, 30, 1, 1, False, "f16"), (256, 8, 64, 16, True, "f32"), (16, 1, 1, 1, False, "f32")]


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("E,K,groups,keep,softmax,dtype", CASES)
def test_weights_of_low_scores(eqb, E, K, groups, keep, softmax, dtype, tied):  # noqa: F811
    say(f"weights of low scores E={E} K={K} groups={groups},{keep} softmax={softmax} {dtype} tied={tied}")
    rng = np.random.default_rng(E + K)
    T, half = 150, E // 2
    z = rng.normal(size=(T, E)) * 1.5
    if tied:                                     # neighbours that are too near to call go through binary64
        z = np.round(z)
    b = np.zeros(E)
    if softmax:
        # the largest logit is an expert's that the bias keeps out of every choice
        z[:, -1] = rng.choice([60.0, 95.0, 100.0, 300.0, 5000.0], size=T)
        b[-1] = -20.0
        if groups > 1:
            b[-(E // groups):] = -20.0
    else:
        z -= rng.choice([0.0, 12.0, 16.0, 60.0, 100.0, 400.0], size=(T, 1))
    if not tied:
        b[:half] += rng.normal(size=half) * 0.1  # the scores are 0 in binary32: the bias alone decides
        b[half:] += rng.normal(size=E - half) * 0.1
    z[7] = -np.inf
    z[8, 1:] = -np.inf
    zt = torch.from_numpy(z).to(torch.float32).to(TYPES[dtype]).cuda()
    z = zt.to(torch.float64).cpu().numpy()
    bt = torch.from_numpy(b.astype(np.float32)).cuda()
    idx, w = torch.full((T, K), -7, dtype=torch.int32, device="cuda"), torch.full((T, K), np.nan, device="cuda")
    score = eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID
    eqb.eqb_route_scored(zt, bt, K, idx, w, score, groups, keep, 2 if E // groups > 1 else 1, True, 2.5)
    g = rng.normal(size=(T, K)).astype(np.float32)
    gz = torch.full((T, E), np.nan, device="cuda")
    eqb.eqb_route_scored_backward(zt, idx, torch.from_numpy(g).cuda(), gz, score, True, 2.5)
    chosen = idx.cpu().numpy()
    assert (chosen[7] == -1).all() and (chosen[8, 1:] == -1).all() and (chosen[np.arange(T) > 8] >= 0).all()
    want, grad, size = want_of(z, chosen, g.astype(np.float64), softmax, 2.5)
    on = chosen >= 0
    x = np.where(on, np.take_along_axis(z, np.maximum(chosen, 0), 1), np.nan)
    x[7] = 0
    d = np.minimum(np.nanmax(x, 1) - np.nanmin(x, 1), 75)[:, None]
    r = (2 * d + 22 + K + 4) * U
    assert (np.abs(w.cpu().numpy() - want) <= r * want + 2.0 ** -100).all()
    assert (np.abs(gz.cpu().numpy() - grad) <= (4 * r + (K + 18) * U) * size + 2.0 ** -100).all()


def test_scores_of_the_lowest_value(eqb):  # noqa: F811
    """Logits of the type's lowest value are no masks: rows of nothing else are rows of equal scores."""
    say("weights of the lowest value")
    for dtype in ("bf16", "f16", "f32"):
        low = float(torch.finfo(TYPES[dtype]).min)
        for softmax in (False, True):
            for E, K in ((8, 2), (64, 8), (256, 12), (64, 20)):
                z = torch.full((5, E), low, dtype=TYPES[dtype])
                z[1, 3] = 0.5
                idx, w = torch.empty((5, K), dtype=torch.int32, device="cuda"), torch.empty((5, K), device="cuda")
                eqb.eqb_route_scored(z.cuda(), None, K, idx, w, eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID)
                got = w.cpu().numpy()
                assert np.abs(got[[0, 2, 3, 4]] - 1 / K).max() <= 4 * U and (idx[0].cpu() == torch.arange(K)).all()
                assert got[1, 0] == 1 and not got[1, 1:].any() and int(idx[1, 0]) == 3
