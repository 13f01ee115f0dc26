"""The oracle of the routing by scores and of the 8-bit products against things it does not go
through: differences, torch's conversions, enumerations and hand-worked cases (CPU)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O


def test_codes_are_torchs():
    """All 256 codes, every code's neighbourhood, the ties between neighbours and random values."""
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(torch.float64).numpy()
    assert np.array_equal(np.isnan(table), np.isnan(O.VALUES)) and np.array_equal(table[~np.isnan(table)], O.VALUES[~np.isnan(table)])
    v = np.sort(table[:127])
    mid = (v[1:] + v[:-1]) / 2
    rng = np.random.default_rng(0)
    y = np.concatenate([v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), rng.uniform(0, 448, 4000), np.exp2(rng.uniform(-14, 8.8, 4000)).clip(0, 448)])
    y = np.concatenate([y, -y]).astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(O.encode(y.astype(np.float64)), want)


def test_exponents_are_the_least():
    for top, x in ((448.0, 0), (448.0001, 1), (449.0, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -126),
                   (2.0 ** -140, -126), (3.4e38, 120), (2.9e38, 119)):
        assert O.exponent(np.array([0.5 * top, -top])) == x, top
        _, s = O.quantize_rows(np.array([[0.5 * top, -top, np.inf, np.nan]]))
        assert s[0, 0] == x + 127, top


def test_rows_columns_and_weights_agree():
    """A block is the same block whichever way it is reached, and decoding is within half a step."""
    rng = np.random.default_rng(1)
    w = rng.normal(size=(2, 200, 300)) * np.exp(rng.normal(size=(2, 200, 1)))
    c, s = O.quantize_weights(w)
    ct, st = O.quantize_weights(w.transpose(0, 2, 1).copy())
    a, b = O.decode_weights(c, s)[:, :, :300], O.decode_weights(ct, st)[:, :, :200]
    assert np.array_equal(a, b.transpose(0, 2, 1))
    step = np.exp2(np.repeat(np.repeat(s[:, :, :3].astype(float) - 127, 128, 1)[:, :200], 128, 2)[:, :, :300])
    assert (np.abs(a - w) <= np.maximum(np.abs(w) * 2.0 ** -4, step * 2.0 ** -10) * (1 + 1e-12)).all()
    offsets = np.array([0, 0, 130, 200])
    W = O.columns(200, offsets)[1]
    cc, cs = O.quantize_columns(w[0], offsets, np.zeros((300, W), np.uint8), np.zeros((300, -(-W // 512) * 4), np.uint8))
    starts, _ = O.columns(200, offsets)
    assert starts == [0, 128, 384] and W == 512
    full = O.decode(cc, cs)
    for e, n in ((1, 130), (2, 70)):
        part = w[0, offsets[e]:offsets[e] + n].T
        assert (np.abs(full[:, starts[e]:starts[e] + n] - part) <= np.abs(part).max(1, keepdims=True) * 2.0 ** -4).all()
        assert not full[:, starts[e] + n:starts[e] + -(-n // 128) * 128].any()


def test_routing_by_hand():
    z = np.log(np.array([[4.0, 1.0, 2.0, 2.0, 1.0, 1.0, 1.0, 3.0]]))
    idx, w = O.route(z, None, 3, softmax=True, normalize=False)
    assert idx.tolist() == [[0, 7, 2]] and np.allclose(w, [[4 / 15, 3 / 15, 2 / 15]])
    idx, w = O.route(z, None, 3, softmax=True, scale=9.0)
    assert np.allclose(w, [[4, 3, 2]])
    # groups of two: sums 5, 4, 2, 4 (of the same two scores): the first and the lower of the equal ones
    v = np.log(np.array([[4.0, 1.0, 2.0, 2.0, 1.0, 1.0, 2.0, 2.0]]))
    idx, w = O.route(v, None, 2, softmax=True, groups=4, top_groups=2, group_top=2)
    assert idx.tolist() == [[0, 2]] and np.allclose(w, [[2 / 3, 1 / 3]])
    # sums 5, 4.5, 2, 4 and largest 4, 2.5, 1, 3
    v = np.log(np.array([[4.0, 1.0, 2.0, 2.5, 1.0, 1.0, 1.0, 3.0]]))
    assert O.route(v, None, 2, softmax=True, groups=4, top_groups=2, group_top=2)[0].tolist() == [[0, 3]]
    assert O.route(v, None, 3, softmax=True, groups=4, top_groups=2, group_top=1)[0].tolist() == [[0, 7, 1]]
    # a bias decides and does not enter the weights
    bias = np.array([0, 0, 0, 0, 5.0, 0, 0, 0])
    idx, w = O.route(z, bias, 2, softmax=True, normalize=False)
    assert idx.tolist() == [[4, 0]] and np.allclose(w, [[1 / 15, 4 / 15]])
    # masks leave one, then none
    z[0, [0, 1, 2, 3, 4, 5, 6]] = -np.inf
    idx, w = O.route(z, None, 3, softmax=True)
    assert idx.tolist() == [[7, -1, -1]] and w.tolist() == [[1, 0, 0]]
    z[0, 7] = -np.inf
    for softmax in (False, True):
        idx, w = O.route(z, bias, 3, softmax=softmax)
        assert idx.tolist() == [[-1, -1, -1]] and not w.any()


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("normalize", [False, True])
def test_route_gradient_is_the_differences(softmax, normalize):
    """Central differences of sum g w with the choice held.  Tolerance: h^2 of third derivatives of order 10 and rounding
    1e-16/h, h = 1e-5."""
    rng = np.random.default_rng(2)
    z, g = rng.normal(size=(4, 8)) * 1.5, rng.normal(size=(4, 3))
    idx, _ = O.route(z, rng.normal(size=8) * 0.2, 3, softmax, normalize=normalize)
    idx[1, 2] = -1
    idx[2, 1] = idx[2, 0]           # the same expert twice
    grad, size = O.route_backward(z, idx, g, softmax, normalize, 2.5)

    def total(v):
        s = O.scores(v, softmax)
        out = 0.0
        for t in range(4):
            on = [k for k in range(3) if idx[t, k] >= 0]
            w = s[t, idx[t, on]]
            out += 2.5 * (g[t, on] @ (w / w.sum() if normalize else w))
        return out

    h = 1e-5
    for t in range(4):
        for e in range(8):
            d = np.zeros_like(z)
            d[t, e] = h
            assert abs((total(z + d) - total(z - d)) / (2 * h) - grad[t, e]) < 1e-8
    assert (np.abs(grad) <= size * (1 + 1e-12)).all()


def test_gated_gradient_is_the_differences():
    rng = np.random.default_rng(3)
    x, gh = rng.normal(size=(3, 10)) * 2, rng.normal(size=(3, 5))
    grad, _ = O.gated_backward(gh, x)
    h = 1e-5
    for i in range(3):
        for j in range(10):
            d = np.zeros_like(x)
            d[i, j] = h
            assert abs(((O.gated(x + d) - O.gated(x - d)) * gh).sum() / (2 * h) - grad[i, j]) < 1e-8
    y = torch.from_numpy(x[:, :5].copy())
    assert np.allclose(O.gated(x), (torch.nn.functional.silu(y).numpy() * x[:, 5:]), atol=1e-15)


def test_planted_mistakes_are_seen():
    """What the checks above would let through if they were vacuous."""
    v = np.log(np.array([[4.0, 1.0, 2.0, 2.5, 1.0, 1.0, 1.0, 3.0]]))
    one, two = (O.route(v, None, 2, softmax=True, groups=4, top_groups=2, group_top=k)[0].tolist() for k in (1, 2))
    assert one != two
    assert O.encode(np.array([17.0]))[0] == O.encode(np.array([16.0]))[0]            # a tie goes to the even code
    assert O.encode(np.array([19.0]))[0] == O.encode(np.array([20.0]))[0]
    assert O.encode(np.array([np.inf]))[0] == 127
