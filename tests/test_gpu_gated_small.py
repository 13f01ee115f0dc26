"""Codes of gated values whose factors or product are subnormal in binary32: bit for bit those of the products in binary64
(their codes are no ties there: the inputs are random or made to miss the ties by a part in 2^17)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_codes import buffers, raw, same_codes
from test_gpu_experts import f64

pytestmark = pytest.mark.gpu


def check(eqb, g, u, dtype=torch.float32, most=0.3):  # noqa: F811
    x = torch.from_numpy(np.concatenate([g, u], 1)).to(dtype).cuda()
    codes, scales = buffers(eqb, (g.shape[0],), g.shape[1])
    eqb.eqb_gated_quantize(x, codes, scales)
    wc, ws = O.quantize_rows(O.gated(f64(x)))
    assert (wc[:, :g.shape[1]] & 127 != 0).mean() > most
    assert np.array_equal(raw(scales), ws) and same_codes(raw(codes), wc)


@pytest.mark.parametrize("F", [7, 128, 200, 1000])
def test_small_gates_of_large_values(eqb, F):  # noqa: F811
    """Gates of few bits (2^-149 to 2^-126): half of one is no number of binary32."""
    say(f"small gates F={F}")
    rng = np.random.default_rng(F)
    R = 64
    g = rng.integers(1, 1 << rng.integers(1, 24, size=(R, F))) * 2.0 ** -149 * rng.choice([-1, 1], size=(R, F))
    for power in (20, 100, 126):
        u = rng.normal(size=(R, F)).clip(-1.9, 1.9) * 2.0 ** power
        check(eqb, g, u)
        ordinary = rng.random((R, 1)) < 0.5          # rows of ordinary gates beside them
        check(eqb, np.where(ordinary, rng.normal(size=(R, F)), g), np.where(ordinary, rng.normal(size=(R, F)), u))
    check(eqb, np.where(rng.random((R, F)) < 0.01, g, 0.0), u, most=0.0)


@pytest.mark.parametrize("F", [5, 130, 600])
def test_small_products(eqb, F):  # noqa: F811
    """Products of 2^-136 (2 j + 1), the middle of two codes in units of the least scale, missed by a fifth of binary32's
    least step: u = n 2^-149, g sigmoid(g) n = 2^13 (2 j + 1) +- 0.2."""
    say(f"small products F={F}")
    rng = np.random.default_rng(F)
    R = 96
    u = rng.integers(20000, 60000, size=(R, F)) * 2.0 ** -149
    odd = 2 * rng.integers(0, 12, size=(R, F)) + 1
    # the gate that meets it, by bisection
    target = (odd * 2 ** 13 + rng.choice([-0.2, 0.2], size=(R, F))) * 2.0 ** -149 * rng.choice([-1, 1], size=(R, F))
    lo, hi = np.full((R, F), 0.01), np.full((R, F), 60.0)
    for _ in range(60):
        mid = (lo + hi) / 2
        up = mid * O.scores(mid, False) * u < np.abs(target)
        lo, hi = np.where(up, mid, lo), np.where(up, hi, mid)
    check(eqb, np.float32(lo).astype(np.float64), u * np.sign(target))
