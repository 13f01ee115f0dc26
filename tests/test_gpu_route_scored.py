"""GPU routing by scores and its gradient against the binary64 oracle.

Tolerances (u = 2^-24).  A sigmoid: exp(-|z|) is the hardware's 2^p (one ulp, 2u) with what p lost put back by one
fma (u), 1 + e is rounded (u), the reciprocal is within an ulp (2u), the product rounded (u): 7u, taken as 8.  A
softmax's exponential: its argument z_max - z = d is rounded once, which is d u of the result, and 3u as above; the sum
over the row, each summand a lane's at most 32nd and then 3 levels (or 8 and 5), is off by what the summands are and 35u,
the quotient 2u.  Of d only what lies within 60 of the largest counts: behind that a term is below e^-60 of the sum.
Weights divide by a sum of K such scores (their error and K u) and are scaled.  Scores below 2^-126 may be 0.
Gradients are products of such scores with differences, whose error is that of the summands: 4 scores' errors
and (K + 10) u of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24


def rel_score(z, softmax):
    if not softmax:
        return 8 * U
    with np.errstate(invalid="ignore"):
        d = (z.max(1, keepdims=True) - z)
    d = np.where(np.isfinite(d), np.minimum(d, 60), 0).max(1, keepdims=True)
    return (2 * d + 45) * U


def make(seed, T, E, dtype, data, bias):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(T, E)) * 1.5 + rng.normal(size=E) * 0.7
    if data == "ties":
        z = np.round(z * 2) / 2
    if data == "masked":
        z[rng.random((T, E)) < 0.4] = -np.inf
        z[rng.random(T) < 0.1] = -np.inf
        if T > 4:
            z[3, 1:] = -np.inf
    if data == "wide":
        z *= 12
    b = {"none": None, "normal": rng.normal(size=E) * 0.1, "steps": np.round(rng.normal(size=E) * 100) / 1000,
         "zero": np.zeros(E), "large": rng.normal(size=E) * 30}[bias]
    zt = torch.from_numpy(z).to(torch.float32).to(TYPES[dtype]).cuda()
    bt = None if b is None else torch.from_numpy(b.astype(np.float32)).cuda()
    return zt, bt


def run(eqb, zt, bt, K, softmax, groups, keep, pair, normalize, scale=2.5):  # noqa: F811
    T = zt.shape[0]
    idx, w = torch.full((T, K), -7, dtype=torch.int32, device="cuda"), torch.full((T, K), np.nan, device="cuda")
    eqb.eqb_route_scored(zt, bt, K, idx, w, eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID, groups, keep, pair,
                         normalize, scale)
    return idx, w


def check(zt, bt, idx, w, K, softmax, groups, keep, pair, normalize, scale=2.5):
    z = zt.to(torch.float64).cpu().numpy()
    b = None if bt is None else bt.cpu().numpy()
    want, ww = O.route(z, b, K, softmax, groups, keep, pair, normalize, scale)
    assert np.array_equal(idx.cpu().numpy(), want)
    r = rel_score(z, softmax)
    tol = ((2 if normalize else 1) * r + (K + 4) * U) * np.abs(ww) + abs(scale) * 2.0 ** -120
    assert (np.abs(w.cpu().numpy() - ww) <= tol).all()
    return want


CASES = [  # T, E, K, groups, keep, pair, dtype, data, bias, softmax, normalize
    (1, 8, 1, 1, 1, 1, "bf16", "normal", "none", False, False), (1, 256, 8, 8, 4, 2, "bf16", "normal", "normal", False, True),
    (7, 8, 7, 1, 1, 2, "f32", "normal", "normal", True, True), (65, 16, 3, 4, 2, 1, "f16", "masked", "steps", False, True),
    (33, 16, 4, 16, 5, 1, "bf16", "normal", "normal", False, True), (40, 32, 8, 8, 3, 2, "bf16", "ties", "none", False, True),
    (300, 32, 5, 2, 1, 2, "f32", "ties", "steps", True, False), (129, 64, 6, 8, 4, 2, "bf16", "boost", "normal", False, True),
    (130, 64, 8, 4, 2, 1, "f16", "masked", "none", True, True), (200, 64, 9, 8, 4, 2, "bf16", "normal", "normal", False, True),
    (77, 128, 8, 8, 3, 2, "bf16", "masked", "normal", True, False), (64, 128, 1, 1, 1, 1, "f32", "normal", "none", False, True),
    (500, 256, 6, 8, 4, 2, "bf16", "normal", "steps", False, True), (501, 256, 8, 1, 1, 1, "bf16", "ties", "zero", False, True),
    (100, 256, 8, 4, 1, 2, "f32", "masked", "normal", True, True), (90, 256, 7, 32, 9, 2, "bf16", "normal", "normal", False, True),
    (50, 256, 16, 16, 4, 2, "f16", "normal", "normal", True, True), (20, 256, 255, 1, 1, 1, "bf16", "normal", "steps", False, True),
    (60, 128, 8, 2, 1, 2, "bf16", "ties", "none", False, True), (40, 256, 8, 8, 4, 2, "bf16", "wide", "none", False, False),
    (60, 64, 4, 64, 10, 1, "bf16", "normal", "large", False, True), (64, 64, 5, 1, 1, 1, "f32", "wide", "normal", True, True),
    (2000, 16, 2, 1, 1, 1, "bf16", "ties", "steps", True, True), (3000, 8, 2, 2, 1, 2, "f16", "ties", "none", False, True)]


@pytest.mark.parametrize("T,E,K,groups,keep,pair,dtype,data,bias,softmax,normalize", CASES)
def test_route(eqb, T, E, K, groups, keep, pair, dtype, data, bias, softmax, normalize):  # noqa: F811
    say(f"route T={T} E={E} K={K} groups={groups},{keep},{pair} {dtype} {data} bias {bias} softmax={softmax} normalize={normalize}")
    zt, bt = make(T + E + K, T, E, dtype, data, bias)
    args = (K, softmax, groups, keep, pair, normalize)
    idx, w = run(eqb, zt, bt, *args)
    want = check(zt, bt, idx, w, *args)

    g = torch.from_numpy(np.random.default_rng(T).normal(size=(T, K)).astype(np.float32)).cuda()
    gz = torch.full((T, E), np.nan, device="cuda")
    eqb.eqb_route_scored_backward(zt, idx, g, gz, eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID, normalize, 2.5)
    z = zt.to(torch.float64).cpu().numpy()
    grad, size = O.route_backward(z, want, g.cpu().numpy().astype(np.float64), softmax, normalize, 2.5)
    tol = (4 * rel_score(z, softmax) + (K + 10) * U) * size + 2.0 ** -115
    assert (np.abs(gz.cpu().numpy() - grad) <= tol).all()


MORE = [  # the same for up to sixteen experts, in lanes of 8, 16 and 32 of them
    (1, 16, 9, 1, 1, 1, "bf16", "normal", "none", False, True), (70, 16, 15, 2, 2, 1, "f32", "masked", "normal", False, True),
    (33, 16, 10, 2, 2, 2, "bf16", "ties", "steps", True, True), (200, 32, 16, 4, 3, 2, "f16", "ties", "none", False, True),
    (129, 64, 10, 4, 2, 2, "bf16", "masked", "steps", False, True), (300, 64, 16, 1, 1, 1, "bf16", "ties", "zero", False, False),
    (90, 128, 9, 8, 3, 2, "f32", "normal", "normal", True, True), (65, 128, 16, 2, 1, 1, "bf16", "masked", "normal", True, False),
    (257, 256, 12, 8, 4, 2, "bf16", "normal", "normal", False, True), (1000, 256, 16, 8, 4, 2, "bf16", "ties", "steps", False, True),
    (64, 256, 16, 1, 1, 1, "f32", "wide", "none", False, True), (100, 256, 13, 4, 1, 2, "f16", "masked", "none", True, True),
    (3, 256, 11, 8, 1, 1, "bf16", "normal", "large", False, True), (400, 256, 17, 8, 4, 2, "bf16", "normal", "normal", False, True)]


@pytest.mark.parametrize("T,E,K,groups,keep,pair,dtype,data,bias,softmax,normalize", MORE)
def test_route_of_more(eqb, T, E, K, groups, keep, pair, dtype, data, bias, softmax, normalize):  # noqa: F811
    say(f"route T={T} E={E} K={K} groups={groups},{keep},{pair} {dtype} {data} bias {bias} softmax={softmax}")
    zt, bt = make(T * 3 + E + K, T, E, dtype, data, bias)
    args = (K, softmax, groups, keep, pair, normalize)
    idx, w = run(eqb, zt, bt, *args)
    check(zt, bt, idx, w, *args)


def test_near_scores_of_more(eqb):  # noqa: F811
    """The K-th and the next of K = 9, 12, 15 and 16, within 2^-26 to 2^-40 of each other."""
    say("near scores of more")
    rng = np.random.default_rng(5)
    T, E = 300, 256
    zt = torch.from_numpy(np.float32(rng.normal(size=(T, E)))).to(torch.bfloat16)
    s = O.scores(zt.to(torch.float64).numpy(), False)
    for trial, K in enumerate((9, 12, 15, 16) * 2):
        b = rng.normal(size=E) * 0.1
        t = trial * 11
        top = np.argsort(-(s[t] + b))
        b[top[40]] += (s[t, top[K]] + b[top[K]]) - (s[t, top[40]] + b[top[40]]) + rng.choice([-1, 1]) * 2.0 ** -rng.integers(26, 40)
        bt = torch.from_numpy(b.astype(np.float32)).cuda()
        for groups, keep in ((1, 1), (8, 5)):
            idx, w = run(eqb, zt.cuda(), bt, K, False, groups, keep, 2, True)
            check(zt, bt, idx, w, K, False, groups, keep, 2, True)


def test_near_scores_are_ordered_as_in_64_bits(eqb):  # noqa: F811
    """Logits and biases made so that score plus bias of two experts differ by 2^-26 to 2^-40, both ways."""
    say("near scores")
    rng = np.random.default_rng(4)
    T, E = 400, 64
    z = np.float32(rng.normal(size=(T, E)))
    zt = torch.from_numpy(z).to(torch.bfloat16)
    s = O.scores(zt.to(torch.float64).numpy(), False)
    # the bias of a random expert of each pair of rows is set so that it meets another's score
    for trial in range(6):
        b = rng.normal(size=E) * 0.1
        t = trial * 7
        top = np.argsort(-(s[t] + b))
        b[top[9]] += (s[t, top[1]] + b[top[1]]) - (s[t, top[9]] + b[top[9]]) + rng.choice([-1, 1]) * 2.0 ** -rng.integers(26, 40)
        bt = torch.from_numpy(b.astype(np.float32)).cuda()
        for K, groups, keep in ((2, 1, 1), (8, 1, 1), (9, 1, 1), (2, 4, 2), (1, 8, 1)):
            idx, w = run(eqb, zt.cuda(), bt, K, False, groups, keep, 2, True)
            check(zt, bt, idx, w, K, False, groups, keep, 2, True)


def test_infinities_and_nan(eqb):  # noqa: F811
    """+inf is the largest score, NaN and -inf are masked out; a bias of NaN or -inf masks its expert, one of +inf leads."""
    say("infinities and NaN")
    for E, K in ((8, 3), (64, 4), (256, 8), (256, 12)):
        z = torch.randn((70, E), generator=torch.Generator().manual_seed(E)).to(torch.bfloat16)
        clean = z.clone()
        z[1, 2], clean[1, 2] = np.nan, -np.inf
        z[2, 1], clean[2, 1] = np.inf, np.inf
        z[3, :] = np.nan
        clean[3, :] = -np.inf
        z[4, 5], clean[4, 5] = -np.inf, -np.inf
        b = torch.zeros(E)
        for bias in (None, b, b.clone()):
            if bias is not None and bias is not b:
                bias[0], bias[3], bias[5] = np.nan, -np.inf, np.inf
            for softmax in (False, True):
                idx, w = run(eqb, z.cuda(), None if bias is None else bias.cuda(), K, softmax, 1, 1, 1, True)
                zz = clean.to(torch.float64).numpy()
                zz[np.isposinf(zz)] = 3.4e38
                if bias is not None and bias is not b:
                    zz[:, [0, 3]] = np.where(np.isneginf(zz[:, [0, 3]]), -np.inf, zz[:, [0, 3]])
                bb = None if bias is None else bias.numpy().astype(np.float64)
                if bb is not None:
                    bb = np.where(np.isnan(bb), -np.inf, bb)
                want, ww = O.route(zz, bb, K, softmax, scale=2.5)
                assert np.array_equal(idx.cpu().numpy(), want), (E, K, softmax)
                got = w.cpu().numpy()
                assert np.isfinite(got).all() and (np.abs(got - ww) <= (2 * 150 * U + (K + 4) * U) * np.abs(ww) + 2.0 ** -120).all()
                gz = torch.full(z.shape, np.nan, device="cuda")
                eqb.eqb_route_scored_backward(z.cuda(), idx, torch.ones((70, K), device="cuda"), gz,
                                              eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID, True, 1.0)
                assert torch.isfinite(gz).all()


def test_gradient_of_given_indices(eqb):  # noqa: F811
    """Indices that no routing gives: outside [0, E), the same one twice and more."""
    say("given indices")
    rng = np.random.default_rng(7)
    T, E, K = 130, 64, 6
    z = torch.from_numpy(rng.normal(size=(T, E)).astype(np.float32)).cuda()
    idx = rng.integers(-3, E + 3, size=(T, K)).astype(np.int32)
    idx[5] = 9
    idx[6, 1:4] = idx[6, 0]
    g = rng.normal(size=(T, K)).astype(np.float32)
    for softmax in (False, True):
        for normalize in (False, True):
            gz = torch.empty((T, E), device="cuda")
            eqb.eqb_route_scored_backward(z, torch.from_numpy(idx).cuda(), torch.from_numpy(g).cuda(), gz,
                                          eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID, normalize, -0.5)
            z64 = z.to(torch.float64).cpu().numpy()
            grad, size = O.route_backward(z64, idx, g.astype(np.float64), softmax, normalize, -0.5)
            tol = (4 * rel_score(z64, softmax) + (K + 10) * U) * size + 2.0 ** -115
            assert (np.abs(gz.cpu().numpy() - grad) <= tol).all()


def test_bit_patterns_streams_and_blocks(eqb):  # noqa: F811
    """BF16 as bit patterns, a stream of its own, capped grids: the same bits."""
    say("streams and blocks")
    zt, bt = make(3, 5000, 128, "bf16", "normal", "normal")
    want = run(eqb, zt, bt, 8, False, 8, 4, 2, True)
    g = torch.randn((5000, 8), device="cuda")
    grad = torch.empty((5000, 128), device="cuda")
    eqb.eqb_route_scored_backward(zt, want[0], g, grad)
    s = torch.cuda.Stream()
    for cap in (1, 3, 0):
        eqb.eqb_set_max_blocks(cap)
        try:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got = run(eqb, zt.view(torch.int16), bt, 8, False, 8, 4, 2, True)
                gz = torch.empty((5000, 128), device="cuda")
                eqb.eqb_route_scored_backward(zt.view(torch.int16), got[0], g, gz)
            s.synchronize()
        finally:
            eqb.eqb_set_max_blocks(0)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(gz, grad)
    eqb.eqb_route_scored(zt[:0], bt, 8, want[0][:0], want[1][:0])
