"""The oracle's normalized weights of scores that binary64 does not hold, against closed forms and differences (CPU)."""
import numpy as np

from oracle import experts_oracle as O


def test_shares_far_below():
    """Far below zero a sigmoid is an exponential, whose ratios do not change with the logits' common part."""
    rng = np.random.default_rng(0)
    z = rng.normal(size=(20, 16))
    bias = rng.normal(size=16)
    for softmax in (False, True):
        for shift in (100.0, 5000.0):
            low = z - shift
            if softmax:                       # the bias keeps the largest logit out
                low = np.concatenate([low, np.zeros((20, 1))], 1)
            b = np.append(bias, -100.0) if softmax else bias
            got_idx, got = O.route(low, b, 4, softmax, scale=2.0)
            x, y = np.take_along_axis(low, got_idx, 1), np.exp(np.take_along_axis(z, got_idx, 1))
            assert (got_idx < 16).all() and (x < -90).all()
            assert np.allclose(got, 2 * y / y.sum(1, keepdims=True), rtol=1e-9)


def test_gradient_far_below_is_the_difference():
    rng = np.random.default_rng(1)
    z, g = rng.normal(size=(6, 8)) - 200, rng.normal(size=(6, 3))
    idx, _ = O.route(z, None, 3)
    grad, size = O.route_backward(z, idx, g)
    assert (np.abs(grad) <= size * (1 + 1e-12)).all()

    def loss(z):
        x = np.take_along_axis(z, idx, 1)
        e = np.exp(x - x.max(1, keepdims=True))
        return (g * e / e.sum(1, keepdims=True)).sum()

    h = 2.0 ** -12
    for t in range(6):
        for e in range(8):
            d = np.zeros_like(z)
            d[t, e] = h
            assert abs(grad[t, e] - (loss(z + d) - loss(z - d)) / (2 * h)) < 1e-6
