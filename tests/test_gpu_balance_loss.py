"""GPU balance loss and its gradient against the binary64 oracle.

Tolerance.  A probability is w / sum w.  The exponential's argument is one binary32
product (|x| log2(e) of it, half an ulp, and the constant's own 1.4e-8) fed to a
hardware exponential and, for a sigmoid, a sum and a hardware reciprocal of an ulp each:
w is off by at most (|x| + 4) 2^-23, relatively; the row's sum by as much, and by
8 roundings; the quotient and product by three more.  So a probability is off by
eps = (2 xmax + 24) 2^-23 at most; a mean of n of them, summed over at most n rows a lane,
by n 2^-24 more; a loss by that and 2^-24.  A gradient is a difference: eps (twice, with the
factor q, once more with sigmoid') times the sum of the magnitudes that it is made of."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


class Case:
    def __init__(self, seed, T, E, K, P=1, mask=False, inf=0.0, scale=1.5, cuts=None, drop=0.0):
        rng = np.random.default_rng(seed)
        x = rng.normal(size=(T, E)) * scale + rng.normal(size=E)
        if inf:
            x[rng.random((T, E)) < inf] = -np.inf
            x[rng.random(T) < inf] = -np.inf                       # rows of nothing
        self.z = bf16(x)
        self.x = self.z.to(torch.float64).numpy()
        self.T, self.E, self.K = T, E, K
        self.idx = np.argsort(-np.where(np.isinf(self.x), -1e30, self.x), axis=1, kind="stable")[:, :K].astype(np.int32)
        self.idx[rng.random((T, K)) < drop] = -1
        self.idx[rng.random((T, K)) < drop / 2] = E
        self.part = [0] + sorted(rng.integers(0, T + 1, size=P - 1).tolist()) + [T] if cuts is None else cuts
        self.P = len(self.part) - 1
        self.valid = (rng.random(T) < 0.8) if mask else None
        self.gl = rng.normal(size=self.P).astype(np.float32)
        self.gs = (rng.normal(size=(T, K)) * 1e-3).astype(np.float32)
        self.inj = (rng.normal(size=(self.P, E)) * 1e-3).astype(np.float32)
        fin = np.abs(self.x[np.isfinite(self.x)])
        self.eps = (2 * (fin.max() if fin.size else 0) + 24) * 2.0 ** -23


def cuda(a, dtype=None):
    return None if a is None else torch.as_tensor(a, dtype=dtype).cuda()


def run(eqb, c, softmax, alpha=0.3, counts=True, router=True, ws=None, valid_type=torch.bool):  # noqa: F811
    score = eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID
    z = c.z.view(torch.int16).cuda()
    idx, valid = cuda(c.idx), cuda(c.valid, valid_type)
    load0 = O.balance_loss(c.x, c.idx, c.K, alpha, c.part, c.valid, softmax)[0]
    load = torch.full((c.P, c.E), -7, dtype=torch.int32, device="cuda") if counts else cuda(load0.astype(np.int32))
    tokens = torch.full((c.P,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((c.P, c.E), float("nan"), device="cuda")
    loss = torch.full((c.P,), float("nan"), device="cuda")
    if ws is None:
        ws = torch.zeros(eqb.eqb_balance_workspace_size(c.E, c.P), dtype=torch.uint8, device="cuda")
    eqb.eqb_balance_loss(z, idx if counts else None, c.K, alpha, load, tokens, prob, loss, ws, valid, c.part, score)
    gz = torch.full((c.T, c.E), float("nan"), device="cuda")
    kw = dict(topk_idx=idx, grad_score=cuda(c.gs), inj=cuda(c.inj)) if router else {}
    eqb.eqb_balance_backward(z, load, tokens, c.K, alpha, cuda(c.gl), gz, valid=valid, part_off=c.part, score=score, **kw)
    torch.cuda.synchronize()
    assert not ws[:1024].any(), "the tickets are zero again"
    return {k: v.cpu().numpy() for k, v in dict(load=load, tokens=tokens, prob=prob, loss=loss, gz=gz).items()}


def check(c, got, softmax, alpha=0.3, router=True):
    load, tokens, prob, loss = O.balance_loss(c.x, c.idx, c.K, alpha, c.part, c.valid, softmax)
    assert np.array_equal(got["load"], load) and np.array_equal(got["tokens"], tokens)
    rel = c.eps + c.T * 2.0 ** -24
    assert np.all(np.abs(got["prob"] - prob) <= rel * prob + 1e-44)
    assert np.all(np.abs(got["loss"] - loss) <= (rel + 2.0 ** -23) * np.abs(loss))
    kw = dict(idx=c.idx, grad_score=c.gs.astype(np.float64), inj=c.inj.astype(np.float64)) if router else {}
    want = O.balance_backward(c.x, load, tokens, c.K, alpha, c.gl.astype(np.float64), c.part, valid=c.valid,
                              softmax=softmax, **kw)
    bound = np.zeros_like(want)
    for p in range(c.P):
        r = slice(c.part[p], c.part[p + 1])
        if tokens[p] == 0:
            continue
        pr = O.probabilities(c.x[r], softmax)
        F = c.E * load[p] / (c.K * tokens[p])
        bound[r] = alpha * abs(float(c.gl[p])) / tokens[p] * pr * (F + (pr @ F)[:, None])
        if router:
            up = np.abs(c.inj[p]).astype(np.float64) + np.zeros_like(pr)
            for k in range(c.K):
                ok = (c.idx[r, k] >= 0) & (c.idx[r, k] < c.E)
                t = np.nonzero(ok)[0]
                up[t, c.idx[r, k][t]] += np.abs(c.gs[r, k][t])
            bound[r] += up * O.sigmoid(c.x[r]) * O.sigmoid(-c.x[r])
    err = np.abs(got["gz"] - want)
    assert np.all(err <= 3 * c.eps * bound + 1e-44), float((err / (bound + 1e-300)).max())
    if c.valid is not None:
        assert np.all(got["gz"][~c.valid] == 0)


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("T,E,K,P,mask,inf", [
    (1, 8, 1, 1, False, 0), (2, 16, 3, 3, False, 0), (63, 8, 7, 2, True, 0.1), (64, 32, 4, 1, False, 0.05),
    (257, 64, 6, 4, True, 0), (300, 128, 16, 5, False, 0.05), (1021, 256, 8, 1, False, 0), (515, 256, 20, 3, True, 0.02),
    (1500, 16, 5, 200, True, 0.05), (3001, 8, 2, 3, False, 0), (130, 256, 255, 2, False, 0), (700, 64, 33, 2, True, 0)])
def test_against_the_oracle(eqb, softmax, T, E, K, P, mask, inf):  # noqa: F811
    say(f"balance T={T} E={E} K={K} P={P} mask={mask} inf={inf} softmax={softmax}")
    c = Case(T * 7 + E, T, E, K, P, mask, inf, drop=0.05 if T > 100 else 0.0)
    check(c, run(eqb, c, softmax), softmax)
    check(c, run(eqb, c, softmax, counts=False, router=False, valid_type=torch.uint8), softmax, router=False)


@pytest.mark.parametrize("E", [8, 64, 256])
def test_rows_far_below_zero(eqb, E):  # noqa: F811
    """Sigmoids that underflow keep their proportions; a mixed batch takes both ways."""
    c = Case(E, 200, E, 2, 2, scale=2.0)
    x = c.z.to(torch.float32)
    x[::3] -= 90.0
    x[1::7] -= 300.0
    c.z = x.to(torch.bfloat16)
    c.x = c.z.to(torch.float64).numpy()
    c.eps = (2 * np.abs(c.x).max() + 24) * 2.0 ** -23
    say(f"balance, rows far below zero, E={E}")
    got = run(eqb, c, False, router=False)
    check(c, got, False, router=False)
    assert np.all(got["prob"] > 0)


def test_empty_groups_and_batches(eqb):  # noqa: F811
    for cuts, T in (([0, 0, 5, 5, 9, 9], 9), ([0, 0, 0], 0), ([0, 0], 0)):
        say(f"balance, groups {cuts}")
        c = Case(3, T, 32, 4, cuts=cuts)
        got = run(eqb, c, False)
        check(c, got, False)
    c = Case(4, 50, 64, 4, P=2, mask=True)
    c.valid[:] = False
    got = run(eqb, c, True)
    check(c, got, True)
    assert not got["loss"].any() and not got["prob"].any() and not got["gz"].any()


def test_what_a_masked_token_holds_does_not_matter(eqb):  # noqa: F811
    """NaN and infinities in the logits and mixture gradients of masked tokens change no bit."""
    c = Case(9, 333, 128, 6, 3, mask=True)
    want = run(eqb, c, False)
    x = c.z.to(torch.float32)
    off = torch.from_numpy(~c.valid)
    x[off] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38] * 32)
    c.z = x.to(torch.bfloat16)
    c.gs[~c.valid] = np.nan
    say("balance, NaN in masked tokens")
    got = run(eqb, c, False)
    for k in want:
        assert np.array_equal(want[k], got[k]), k


def test_blocks_and_repeats(eqb):  # noqa: F811
    """Any number of blocks gives the result within the tolerance, and the same call the same bits; one workspace
    serves call after call."""
    c = Case(11, 5003, 64, 6, 7, mask=True, drop=0.02)
    ws = torch.zeros(eqb.eqb_balance_workspace_size(c.E, c.P), dtype=torch.uint8, device="cuda")
    first = run(eqb, c, False, ws=ws)
    for cap in (1, 3, 7, 0, 0):
        say(f"balance, at most {cap} blocks")
        eqb.eqb_set_max_blocks(cap)
        try:
            got = run(eqb, c, False, ws=ws)
        finally:
            eqb.eqb_set_max_blocks(0)
        check(c, got, False)
    for k in first:
        assert np.array_equal(first[k], got[k]), k


def test_agrees_with_the_router_backward(eqb):  # noqa: F811
    """With alpha = 0 the gradient is eqb_lei_router_backward's, to the tolerance of both (eps and 3e-7)."""
    c = Case(12, 2000, 256, 8, 2)
    got = run(eqb, c, False, alpha=0.0)["gz"]
    gz = torch.empty((c.T, c.E), device="cuda")
    eqb.eqb_lei_router_backward(c.z.view(torch.int16).cuda(), cuda(c.idx), cuda(c.gs), gz, cuda(c.inj), c.part)
    want = gz.cpu().numpy()
    assert np.all(np.abs(got - want) <= (c.eps + 3e-7) * np.abs(want) + 1e-44)


def test_gradient_is_the_differences(eqb):  # noqa: F811
    """The device's losses at logits moved by h against its gradient: for a direction d over all logits the
    difference quotient and <grad, d> agree to h^2 (third derivatives below 1) and the losses' rounding over 2h
    (alpha 1 of losses near 1, each off by eps)."""
    T, E, K, P = 64, 16, 3, 2
    c = Case(13, T, E, K, P, scale=0.5)
    c.gl[:] = 1.0
    rng = np.random.default_rng(1)
    h = 2.0 ** -3
    # logits in steps of 2^-6 near 1: moving them by h is exact in BF16
    base = np.round(c.x.clip(-1, 1) * 64) / 64
    d = rng.integers(-1, 2, size=(T, E)).astype(np.float64)
    losses = []
    for s in (h, -h, 0.0):
        c.x = base + s * d
        c.z = bf16(c.x)
        assert np.array_equal(c.z.to(torch.float64).numpy(), c.x)
        c.eps = (2 * 2 + 24) * 2.0 ** -23
        losses.append(run(eqb, c, True, alpha=1.0, router=False))
    quotient = (losses[0]["loss"].astype(np.float64).sum() - losses[1]["loss"].sum()) / (2 * h)
    slope = float((losses[2]["gz"] * d).sum())
    assert abs(quotient - slope) <= h * h + P * 4 * c.eps / (2 * h)


def test_on_another_stream(eqb):  # noqa: F811
    c = Case(14, 3000, 128, 4, 2)
    want = run(eqb, c, False)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = run(eqb, c, False)
    for k in want:
        assert np.array_equal(want[k], got[k])


def test_large_batch(eqb):  # noqa: F811
    """Past 2^32 bytes of logits, of copies of one piece: the means are the piece's, every count is as many times its
    own, and rows far into the batch have their copy's gradient, scaled by the group's size."""
    n, E, K, copies = 65536, 256, 8, 131
    c = Case(15, n, E, K)
    say("balance, 8.6 M tokens")
    z1 = c.z.view(torch.int16).cuda()
    z = z1.repeat(copies, 1)
    idx = cuda(c.idx).repeat(copies, 1)
    T = n * copies
    load = torch.empty((1, E), dtype=torch.int32, device="cuda")
    tokens, loss, prob = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, device="cuda"), torch.empty((1, E), device="cuda")
    ws = torch.zeros(eqb.eqb_balance_workspace_size(E, 1), dtype=torch.uint8, device="cuda")
    gz = torch.empty((T, E), device="cuda")
    eqb.eqb_balance_loss(z, idx, K, 0.5, load, tokens, prob, loss, ws)
    eqb.eqb_balance_backward(z, load, tokens, K, 0.5, torch.ones(1, device="cuda"), gz)
    load1, tokens1, prob1, loss1 = O.balance_loss(c.x, c.idx, K, 0.5, [0, n])
    assert np.array_equal(load.cpu().numpy(), copies * load1) and int(tokens) == T
    rel = c.eps + 8192 * 2.0 ** -24             # a lane sums T / 256 blocks / 32 rows
    assert np.all(np.abs(prob.cpu().numpy() - prob1) <= rel * prob1)
    assert abs(float(loss) - loss1[0]) <= 2 * rel * loss1[0]
    want = O.balance_backward(c.x[:64], load1, tokens1, K, 0.5, [1.0], [0, 64]) / copies
    F = E * load1[0] / (K * n)
    pr = O.probabilities(c.x[:64], False)
    bound = 0.5 / T * pr * (F + (pr @ F)[:, None])
    for k in (0, 65, 130):
        got = gz[k * n:k * n + 64].cpu().numpy()
        assert np.all(np.abs(got - want) <= 3 * c.eps * bound + 1e-44)


@pytest.mark.parametrize("K", [1, 2, 3, 7, 16, 100, 255])
def test_masked_counts(eqb, K):  # noqa: F811
    """The counts of masked batches, every fan-out: a pair's token is found by a product with K's reciprocal."""
    T, E = 70001 if K < 16 else 9001, 256
    g = torch.Generator(device="cuda")
    g.manual_seed(K)
    d = dict(device="cuda")
    z = torch.randn((T, E), generator=g, **d).to(torch.bfloat16).view(torch.int16)
    idx = torch.randint(-2, E + 2, (T, K), generator=g, **d).to(torch.int32)
    valid = torch.rand(T, generator=g, **d) < 0.7
    cuts = [0, 11, T // 3, T // 3, T]
    load, tokens = torch.empty((4, E), dtype=torch.int32, **d), torch.empty(4, dtype=torch.int32, **d)
    ws = torch.zeros(eqb.eqb_balance_workspace_size(E, 4), dtype=torch.uint8, **d)
    say(f"balance, masked counts K={K}")
    for score in (eqb.EQB_SCORE_SIGMOID, eqb.EQB_SCORE_SOFTMAX):
        eqb.eqb_balance_loss(z, idx, K, 1.0, load.fill_(-1), tokens, torch.empty((4, E), **d), torch.empty(4, **d), ws, valid,
                             cuts, score)
        for p, (a, b) in enumerate(zip(cuts, cuts[1:])):
            mine = idx[a:b][valid[a:b]]
            mine = mine[(mine >= 0) & (mine < E)].long()
            assert torch.equal(load[p].long(), torch.bincount(mine.reshape(-1), minlength=E)), p
            assert int(tokens[p]) == int(valid[a:b].sum())


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("E", [8, 128, 256])
def test_masks_of_the_lowest_value(eqb, E, softmax):  # noqa: F811
    """Experts masked by BF16's lowest value instead of -inf: 0 beside others, and a row of nothing else is a row of
    equal logits (probabilities 1/E)."""
    c = Case(E, 90, E, 2, 2)
    x = c.z.to(torch.float32)
    low = torch.finfo(torch.bfloat16).min
    x[::3, 1::2] = low
    x[1::5] = low
    x[2::7, :E // 2] = -float("inf")
    x[4] = -float("inf")
    x[5] = low
    x[5, 3] = -float("inf")
    c.z = x.to(torch.bfloat16)
    c.x = c.z.to(torch.float64).numpy()
    # the masked entries' own rounding does not count: their weights are 0 or 1 exactly
    c.eps = (2 * np.abs(c.x[np.abs(c.x) < 1e30]).max() + 24) * 2.0 ** -23
    say(f"balance, lowest values E={E} softmax={softmax}")
    got = run(eqb, c, softmax, router=False)
    assert np.all(np.isfinite(got["gz"])) and np.all(np.isfinite(got["prob"]))
    check(c, got, softmax, router=False)


@pytest.mark.parametrize("E,K,router", [(256, 8, True), (128, 4, False), (8, 4, True)])
@pytest.mark.parametrize("softmax", [False, True])
def test_gradient_of_a_large_batch(eqb, E, K, router, softmax):  # noqa: F811
    """Logits that the memory-side cache does not keep take other loads; a row's gradient is the same in a batch of
    half the size."""
    T = (1 << 25) // E + 777
    g = torch.Generator(device="cuda")
    g.manual_seed(E)
    d = dict(device="cuda")
    z = torch.randn((T, E), generator=g, **d).to(torch.bfloat16).view(torch.int16)
    valid = torch.rand(T, generator=g, **d) < 0.9
    load = torch.randint(0, T, (1, E), generator=g, **d).int()
    tokens, one = torch.full((1,), T, dtype=torch.int32, **d), torch.ones(1, **d)
    pairs = {}
    if router:
        pairs = dict(topk_idx=torch.arange(T * K, **d).view(T, K).remainder_(E).int(),
                     grad_score=torch.randn((T, K), generator=g, **d))
    inj = dict(inj=torch.randn((1, E), generator=g, **d)) if router else {}
    say(f"balance gradient T={T} E={E} K={K} router={router} softmax={softmax}")
    kw = dict(score=eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID)
    whole, half = torch.full((T, E), 7.0, **d), torch.empty((T // 2, E), **d)
    eqb.eqb_balance_backward(z, load, tokens, K, 1e-2, one, whole, valid=valid, **pairs, **inj, **kw)
    eqb.eqb_balance_backward(z[:T // 2], load, tokens, K, 1e-2, one, half, valid=valid[:T // 2],
                             **{n: t[:T // 2] for n, t in pairs.items()}, **inj, **kw)
    assert torch.equal(whole[:T // 2], half)
    eqb.eqb_balance_backward(z[-(T // 2):], load, tokens, K, 1e-2, one, half, valid=valid[-(T // 2):],
                             **{n: t[-(T // 2):] for n, t in pairs.items()}, **inj, **kw)
    assert torch.equal(whole[-(T // 2):], half)
    assert bool((whole[~valid] == 0).all())
