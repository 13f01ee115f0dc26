"""Gated values that F16 cannot hold: the codes that the second product takes hold them, and so do those that the
gradient of its weights takes.

Tolerance of the gradient of down: a code is within 2^-4 of its value or, below the normal codes, within half of their
step, 2^-10 of the block's scale, which is less than top / 224; a value that fits the type is rounded to it first (F16: 2^-11).
The gradient sums products of two such, in binary32: 128 B 2^-24 of their magnitudes for B blocks."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from paper_2609_28053_amd import ExpertRows, GatedExperts
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_codes import buffers, raw, same_codes
from test_gpu_experts import TYPES, away, f64

pytestmark = pytest.mark.gpu
D = dict(device="cuda")


def test_gradient_of_down_where_gated_values_overflow():
    say("gated values beyond F16")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    T, E, K, H, F = 200, 8, 2, 96, 40
    x = torch.randn((T, H), generator=g, **D).to(torch.float16)
    up = torch.randn((E, 2 * F, H), generator=g, **D) * H ** -0.5
    up[:, [3, 17]] *= 400                       # gates of some 400 and their u's of some 300
    up[:, [F + 3, F + 17]] *= 300
    down = torch.randn((E, H, F), generator=g, **D) * 1e-3
    down[:, :, [3, 17]] *= 1e-3
    rows, experts = ExpertRows(T, E, K), GatedExperts(up.to(torch.float16), down.to(torch.float16))
    idx = torch.stack([torch.randperm(E, generator=g, **D)[:K] for _ in range(T)]).to(torch.int32)
    rows.plan(idx)
    out, saved = experts.forward(x, rows)
    grad_out = torch.randn((T * K, H), generator=g, **D).to(torch.float16)
    grad_rows, grad_up, grad_down = experts.backward(grad_out, saved)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(grad_down).all())
    h = O.gated(f64(saved[1]))
    assert (np.abs(h) > 65504).any() and np.isfinite(h).all()
    off = rows.offsets.cpu().numpy()
    gout, got = f64(grad_out), f64(grad_down)
    for e in range(E):
        p, q = gout[off[e]:off[e + 1]], h[off[e]:off[e + 1]]
        pa, qa = np.abs(p), np.abs(q)
        # half a code's step of the columns' least codes
        pe, qe = pa * 2.0 ** -4 + pa.max(0) / 224 * 2.0 ** -10, qa * (2.0 ** -4 + 2.0 ** -11 + 2.0 ** -14) + qa.max(0) / 224 * 2.0 ** -10
        most = (pa + pe).T @ (qa + qe)
        blocks = -(-p.shape[0] // 128)
        tol = most - pa.T @ qa + 128 * blocks * 2.0 ** -24 * most
        assert (np.abs(got[e] - p.T @ q) <= tol).all()


COUNTS = [[1], [0, 0, 5], [128, 0, 1, 127, 129], [0], [3] * 40, [700]]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
def test_gated_columns(eqb, dtype, counts):  # noqa: F811
    """Bit for bit the columns' codes of what eqb_gated stores."""
    rng = np.random.default_rng(sum(counts))
    for H, behind in ((1, 3), (130, 7), (200, 260)):
        R = sum(counts) + behind
        say(f"gated columns {len(counts)} experts, {R} rows of {H} {dtype}")
        x = away((R, 2 * H), TYPES[dtype], rng, H % 2, 3.0)
        offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
        W = eqb.eqb_column_width(R, len(counts))
        codes, scales = buffers(eqb, (H,), W)
        eqb.eqb_gated_quantize_columns(x, offsets, codes, scales)
        h = torch.empty((R, H), dtype=TYPES[dtype], **D)
        eqb.eqb_gated(x, h)
        want, wants = buffers(eqb, (H,), W)
        eqb.eqb_quantize_columns(h, offsets, want, wants)
        assert np.array_equal(raw(codes), raw(want)) and np.array_equal(raw(scales), raw(wants))


def test_gated_columns_beyond_f16(eqb):  # noqa: F811
    """Gates from 32 on have a sigmoid of 1, and integers of up to 11 bits a product that binary32 holds: the codes are the
    oracle's of the products, rounded to F16 where that holds them.  Rows that are no numbers stay that."""
    say("gated columns beyond F16")
    rng = np.random.default_rng(2)
    R, H = 300, 70
    g, u = rng.integers(32, 1500, size=(R, H)).astype(np.float64), rng.integers(-1500, 1500, size=(R, H)).astype(np.float64)
    g[5, 3], u[6, 4], u[7, 5] = np.nan, np.nan, np.inf
    h = g * u
    with np.errstate(over="ignore", invalid="ignore"):
        f16 = h.astype(np.float16).astype(np.float64)
    h = np.where(np.isfinite(f16), f16, h)
    assert (np.abs(h[np.isfinite(h)]) > 65504).mean() > 0.5
    off = np.array([0, 130, 130, 300], np.int32)
    x = torch.from_numpy(np.concatenate([g, u], 1)).to(torch.float16).cuda()
    codes, scales = buffers(eqb, (H,), eqb.eqb_column_width(R, 3))
    wc, ws = O.quantize_columns(h, off, raw(codes).copy(), raw(scales).copy())
    eqb.eqb_gated_quantize_columns(x, torch.from_numpy(off).cuda(), codes, scales)
    assert same_codes(raw(codes), wc) and np.array_equal(raw(scales), ws)


def test_large_gated_columns(eqb):  # noqa: F811
    """Gates of more than 256 MiB, which pass the caches by."""
    say("large gated columns")
    x = torch.randn((70000, 2 * 1024), generator=torch.Generator(device="cuda").manual_seed(3), dtype=torch.bfloat16, **D)
    offsets = torch.tensor([0, 20001, 20001, 69900], dtype=torch.int32, **D)
    got, want = ([*buffers(eqb, (1024,), eqb.eqb_column_width(70000, 3))] for _ in range(2))
    eqb.eqb_gated_quantize_columns(x, offsets, *got)
    h = torch.empty((70000, 1024), dtype=torch.bfloat16, **D)
    eqb.eqb_gated(x, h)
    eqb.eqb_quantize_columns(h, offsets, *want)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    eqb.eqb_gated_quantize_columns(x[:0], torch.zeros(4, dtype=torch.int32, **D), *buffers(eqb, (1024,), eqb.eqb_column_width(0, 3)))
