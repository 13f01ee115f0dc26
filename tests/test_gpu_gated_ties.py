"""Codes of gated values near the middle of two: bit for bit those of the exact products.

For a gate near 0 the sigmoid is 1/2 and a little, g sigmoid(g) u is g u / 2 and a little, and g u / 2 of BF16 numbers has
few bits: it often is the middle of two codes, from which the little leads away.

Reference: p + p tanh(g / 2), p = g u / 2, in numpy's longdouble of 64 bits (p is exact: 24 + 24 bits), moved by its last bit
where that does not hold the second term (|g| below 2^-63; codes have 4 bits and p at most 48, so that no middle is passed)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_codes import buffers, raw, same_codes
from test_gpu_experts import f64

pytestmark = pytest.mark.gpu


def exact(x):
    assert np.finfo(np.longdouble).nmant >= 63
    g, u = np.split(x.astype(np.longdouble), 2, axis=1)
    p = g * u / 2
    t = p * np.tanh(g / 2)
    h = np.where(t == 0, p, p + t)               # a zero keeps its sign: -0 and +0 would be +0
    return np.where((h == p) & (t != 0), np.nextafter(p, np.where(t > 0, np.inf, -np.inf).astype(np.longdouble)), h)


def check(eqb, g, u, dtype):  # noqa: F811
    x = torch.from_numpy(np.concatenate([g, u], 1)).to(dtype).cuda()
    codes, scales = buffers(eqb, (g.shape[0],), g.shape[1])
    eqb.eqb_gated_quantize(x, codes, scales)
    wc, ws = O.quantize_rows(exact(f64(x)))
    assert (wc[:, :g.shape[1]] & 127 != 0).mean() > 0.3
    assert np.array_equal(raw(scales), ws) and same_codes(raw(codes), wc)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_small_gates_on_the_middle(eqb, dtype):  # noqa: F811
    """g a power of two, u of five bits, the last one set: g u / 2 is the middle of two codes."""
    say(f"small gates on the middle {dtype}")
    rng = np.random.default_rng(8)
    R, F = 400, 130
    most = 14 if dtype == "f16" else 120
    g = np.exp2(-rng.integers(2, most, size=(R, F))) * rng.choice([-1, 1], size=(R, F))
    u = (2 * rng.integers(8, 16, size=(R, F)) + 1) * rng.choice([-1, 1], size=(R, F)) / np.abs(g) * np.exp2(rng.integers(-4, 1, size=(R, F)))
    if dtype == "f16":
        u = np.where(np.abs(u) < 65504, u, 1.0)
    else:
        assert np.abs(u).max() < 3e38
    check(eqb, g, u, {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[dtype])


def test_far_gates_are_zero(eqb):  # noqa: F811
    """Gates of any size below -1,000 give 0, whatever u is."""
    say("far gates")
    g = torch.tensor([[-1e3, -2e3, -1e10, -1e30, -3e38, 1.0]], device="cuda")
    for far in (g, g[:, [3, 4, 0, 1, 2, 5]]):
        u = torch.tensor([[3e38, 3e38, -3e38, 3e38, -3e38, 1e-30]], device="cuda")
        codes, scales = buffers(eqb, (1,), 6)
        eqb.eqb_gated_quantize(torch.cat([far, u], 1), codes, scales)
        got = O.decode(raw(codes), raw(scales))[0]
        assert not got[:5].any() and abs(got[5] - 1e-30 / (1 + np.exp(-1.0))) < 2.0 ** -4 * 1e-30


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_small_numbers(eqb, dtype):  # noqa: F811
    """Rows of every size from the least number up, and rows of zeros."""
    say(f"rows of small numbers {dtype}")
    rng = np.random.default_rng(3)
    R, F = 300, 300
    g = rng.normal(size=(R, F)) * np.exp2(rng.integers(-149, 3, size=(R, 1)))
    u = rng.normal(size=(R, F)) * np.exp2(rng.integers(-149, 100, size=(R, 1)))
    keep = np.abs(g * u).max(1) > 2.0 ** -134
    check(eqb, g[keep], u[keep], torch.bfloat16 if dtype == "bf16" else torch.float32)
    x = torch.zeros((4, 600), dtype=torch.bfloat16, device="cuda")
    codes, scales = buffers(eqb, (4,), 300)
    eqb.eqb_gated_quantize(x, codes, scales)
    assert not raw(codes).any() and (raw(scales)[:, :3] == 1).all()
