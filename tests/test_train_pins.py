"""The oracle of the training operators against things it does not go through: differences,
enumerations, published code points and hand-worked cases (CPU)."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as O


def logits(seed, T, E, inf=0.0):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(T, E)) * 1.5 + rng.normal(size=E)
    if inf:
        x[rng.random((T, E)) < inf] = -np.inf
    return x


@pytest.mark.parametrize("softmax", [False, True])
def test_gradient_is_the_differences(softmax):
    """d(sum_p gl_p loss_p + sum g s_sel + sum inj s)/dz by central differences with the loads held.  Tolerance:
    the second-order error h^2/6 of terms below 1, and rounding 1e-16/h, h = 1e-5."""
    T, E, K, alpha = 6, 8, 3, 0.7
    part = [0, 4, 4, 6]
    rng = np.random.default_rng(5)
    x = logits(1, T, E)
    idx = np.argsort(-x, axis=1)[:, :K].copy()
    idx[2, 1] = -1
    valid = np.array([1, 1, 0, 1, 1, 1], dtype=bool)
    gl, gs, inj = rng.normal(size=3), rng.normal(size=(T, K)), rng.normal(size=(3, E))
    load, tokens, _, _ = O.balance_loss(x, idx, K, alpha, part, valid, softmax)

    def total(v):
        _, _, _, loss = O.balance_loss(v, None, K, alpha, part, valid, softmax, load=load)
        s = 1 / (1 + np.exp(-v))
        out = float(gl @ loss)
        for t in range(T):
            if not valid[t]:
                continue
            p = 0 if t < 4 else 2
            out += float(inj[p] @ s[t]) + sum(gs[t, k] * s[t, idx[t, k]] for k in range(K) if idx[t, k] >= 0)
        return out

    got = O.balance_backward(x, load, tokens, K, alpha, gl, part, idx, gs, inj, valid, softmax)
    h = 1e-5
    for t, e in np.ndindex(T, E):
        up, down = x.copy(), x.copy()
        up[t, e] += h
        down[t, e] -= h
        assert abs((total(up) - total(down)) / (2 * h) - got[t, e]) < 1e-9
    assert np.all(got[2] == 0)


def test_even_load_costs_alpha_and_all_on_one_costs_more():
    """Equal probabilities and loads: alpha.  All of K = 1 on expert 0 with probability near 1: alpha E."""
    T, E = 16, 8
    idx = (np.arange(T) % E)[:, None]
    load, tokens, prob, loss = O.balance_loss(np.zeros((T, E)), idx, 1, 0.5, [0, T])
    assert np.all(load == 2) and tokens[0] == T
    assert np.allclose(prob, 1 / E, rtol=1e-14) and np.allclose(loss, 0.5, rtol=1e-14)
    x = np.full((T, E), -40.0)
    x[:, 0] = 40.0
    for softmax in (False, True):
        assert np.allclose(O.balance_loss(x, np.zeros((T, 1), dtype=int), 1, 0.5, [0, T], None, softmax)[3], 0.5 * E)


def test_masked_rows():
    """-inf has probability 0, a row of -inf none at all, and sigmoids that underflow binary32 keep their proportions."""
    x = np.array([[0.0, -np.inf, 0.0, -np.inf], [-np.inf] * 4, [-200.0, -201.0, -np.inf, -200.0]])
    for softmax in (False, True):
        p = O.probabilities(x, softmax)
        assert np.allclose(p[0], [0.5, 0, 0.5, 0]) and np.all(p[1] == 0)
        e = np.exp(-1.0)
        assert np.allclose(p[2], np.array([1, e, 0, 1]) / (2 + e))
    load, tokens, prob, loss = O.balance_loss(x, np.array([[0], [1], [-1]]), 1, 1.0, [0, 3], [False] * 3)
    assert tokens[0] == 0 and loss[0] == 0 and np.all(prob == 0) and np.all(load == 0)


def test_plan_is_the_stable_sort():
    rng = np.random.default_rng(2)
    idx = rng.integers(-1, 9, size=(23, 3))             # -1 and 8 lie outside
    offsets, slot = O.dispatch_plan(idx, 8)
    flat = idx.reshape(-1)
    inside = np.nonzero((flat >= 0) & (flat < 8))[0]
    order = inside[np.argsort(flat[inside], kind="stable")]
    want = np.full(flat.size, -1)
    want[order] = np.arange(order.size)
    assert np.array_equal(slot.reshape(-1), want)
    assert np.array_equal(offsets, np.searchsorted(flat[order], np.arange(9)))


def test_rows_gradients_are_the_adjoints():
    """<dispatch(x), r> = <x, combine(r)> without weights; combine's gradients by linearity in rows and weights."""
    rng = np.random.default_rng(3)
    T, K, H, R = 7, 2, 5, 14
    slot = rng.permutation(R).reshape(T, K)
    slot[1, 0] = -1
    x, r, gy, w = rng.normal(size=(T, H)), rng.normal(size=(R, H)), rng.normal(size=(T, H)), rng.normal(size=(T, K))
    assert np.isclose((O.dispatch(x, slot, np.zeros((R, H))) * r).sum(), (x * O.combine(r, slot, None, H)).sum())
    gr, gw = O.combine_backward(gy, r, slot, w, np.zeros((R, H)))
    d = rng.normal(size=(R, H))
    assert np.isclose((gr * d).sum(), (gy * O.combine(d, slot, w, H)).sum())
    dw = rng.normal(size=(T, K))
    assert np.isclose((gw * dw).sum(), (gy * O.combine(r, slot, dw, H)).sum())


def test_e4m3_values_are_the_formats():
    """The decoded codes against torch's own type, and the format's end points."""
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(O.E4M3, want, equal_nan=True)
    assert O.E4M3[0x7E] == 448 and O.E4M3[1] == 2.0 ** -9 and O.E4M3[8] == 2.0 ** -6


def test_random_rounding_is_right_on_average():
    """Over all 2^16 random numbers a value between two codes is rounded up by its exact share (to 2^-16)."""
    rnd = np.arange(65536)
    for y in (0.0, 2.0 ** -9, 2.0 ** -10, 2.0 ** -6 * 0.99, 2.0 ** -6, 1.03, 447.9, 448.0, 100.0 / 3):
        c = O.round_e4m3(np.full(65536, y), rnd)
        lo, hi = O.E4M3[c.min()], O.E4M3[c.max()]
        assert lo <= y <= hi and c.max() - c.min() <= 1
        assert abs(O.E4M3[c].mean() - y) <= (hi - lo) / 65536 + 1e-12


def test_random_bits_are_spread():
    """Both halves of the random bits: mean and variance of a uniform 16-bit number (five standard errors), and no
    correlation between neighbours, halves, tensors or steps."""
    n = 1 << 16
    r = O.random32(n, O.tensor_key(1, 1, 0))
    for x in (r & 0xFFFF, r >> 16):
        assert abs(x.mean() - 32767.5) < 5 * 65536 / np.sqrt(12 * n)
        assert abs(x.var() / (65536 ** 2 / 12) - 1) < 5 * np.sqrt(0.8 / n)
    others = [np.roll(r, 1), O.random32(n, O.tensor_key(1, 2, 0)), O.random32(n, O.tensor_key(1, 1, 1)),
              O.random32(n, O.tensor_key(2, 1, 0))]
    for o in others:
        assert abs(np.corrcoef(r & 0xFFFF, o & 0xFFFF)[0, 1]) < 5 / np.sqrt(n)
        assert abs(np.corrcoef(r >> 16, o >> 16)[0, 1]) < 5 / np.sqrt(n)
    assert abs(np.corrcoef(r >> 16, r & 0xFFFF)[0, 1]) < 5 / np.sqrt(n)


def test_adamw_against_torch():
    """Five steps of torch.optim.AdamW in binary64 (another implementation of the same update)."""
    rng = np.random.default_rng(4)
    w = rng.normal(size=50)
    p = torch.nn.Parameter(torch.from_numpy(w.copy()))
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.9), eps=1e-6, weight_decay=0.3)
    m = v = np.zeros(50)
    for step in range(1, 6):
        g = rng.normal(size=50)
        p.grad = torch.from_numpy(g.copy())
        opt.step()
        w, m, v = O.adamw(w, g, m, v, step, 1e-2, 0.8, 0.9, 1e-6, 0.3)
        assert np.allclose(w, p.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_quantised_blocks():
    """A block's largest value is exact, a small second moment keeps a code above 0, an empty block is all 0, a short
    last block stands alone."""
    x = np.zeros(2 * O.BLOCK + 3)
    x[:O.BLOCK] = np.linspace(-1, 1, O.BLOCK)
    x[-3:] = [1e-3, -2e-3, 5e-10]
    codes, scales = O.quantise(x, np.zeros(len(x), dtype=np.int64), True)
    back = O.dequantise(codes, scales)
    assert back[0] == -1.0 and np.isclose(back[-2], -2e-3, rtol=1e-15) and scales[1] == 0
    assert np.all(back[O.BLOCK:2 * O.BLOCK] == 0) and back[-1] > 0
    assert np.all(np.abs(back - x)[:O.BLOCK] <= np.abs(x)[:O.BLOCK] / 8 + scales[0] * 2.0 ** -9)


def test_planted_mistakes_are_seen():
    """Mistakes planted in the oracle's own formulas move the results by far more than the tolerances used."""
    x = logits(7, 12, 8)
    idx = np.argsort(-x, axis=1)[:, :2]
    load, tokens, prob, loss = O.balance_loss(x, idx, 2, 1.0, [0, 12])
    s = O.sigmoid(x)
    assert abs(loss[0] - float((4 * load[0] / 12 * s.mean(0)).sum())) > 1e-2          # sigmoids not normalised
    g = O.balance_backward(x, load, tokens, 2, 1.0, [1.0], [0, 12])
    p = O.probabilities(x, False)
    assert np.abs(g - p * (4 * load[0] / 12) / 12 * O.sigmoid(-x)).max() > 1e-3       # without the mean taken off
    w = O.adamw(np.ones(3), np.ones(3), np.zeros(3), np.zeros(3), 1, 0.1, 0.9, 0.999, 1e-8, 0.1)[0]
    assert np.allclose(w, 1 - 0.01 - 0.1, atol=1e-7) and not np.allclose(w, 1 - 0.1 * (1 + 0.1 * 0.9), atol=1e-4)
