"""GPU products of 8-bit codes against products in binary64 of what the codes stand for.

Tolerance.  A block of 128 contributes sum_k p_k q_k times a power of two.  For results of 16 bits the
matrix instruction cuts each product off at 2^-16 of the block's largest product: at most 128 2^-16 = 2^-9
of the largest a block; adding the blocks in binary32 rounds each sum once, B 2^-24 of the magnitudes' sum;
then half an ulp of the type.  For results in binary32 products are exact and every addition, of up to B 128
terms in any order, rounds once: 128 B 2^-24 of the magnitudes' sum at the very most (and a code times its
scale below 2^-133 is lost, which these inputs have not)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_experts import HALF_ULP, STEP, TYPES

pytestmark = pytest.mark.gpu
BLOCK = 128


def coded(eqb, rng, lead, hidden, spread=1.0):  # noqa: F811
    """Random codes of rows [lead, hidden] with random powers, as a user would hold them, and their values."""
    W, S = eqb.eqb_code_width(hidden), eqb.eqb_scale_width(hidden)
    codes = torch.randint(0, 256, (lead, W), generator=rng, device="cuda", dtype=torch.uint8)
    codes = torch.where((codes & 127) == 127, codes - 1, codes)
    codes[:, hidden:] = 0
    scales = (127 + spread * torch.randn((lead, S), generator=rng, device="cuda")).round().clamp(1, 250).to(torch.uint8)
    return codes, scales


def values(codes, scales):
    v = codes.view(torch.float8_e4m3fn).to(torch.float64)
    return v * torch.exp2(scales.to(torch.float64) - 127).repeat_interleave(BLOCK, 1)[:, :v.shape[1]]


def bound(p, q, dtype):
    """The tolerance of p q^T before the type's rounding (p [n,W], q [m,W])."""
    blocks = p.shape[1] // BLOCK
    size = p.abs() @ q.abs().t()
    if dtype == "f32":
        return 128 * blocks * 2.0 ** -24 * size
    cut = torch.zeros_like(size)
    for b in range(blocks):
        pb, qb = p[:, b * BLOCK:(b + 1) * BLOCK].abs(), q[:, b * BLOCK:(b + 1) * BLOCK].abs()
        # at least the largest product: the largest of one with the largest of the other
        cut += 2.0 ** -9 * pb.amax(1)[:, None] * qb.amax(1)[None]
    return cut + blocks * 2.0 ** -24 * size


def close(got, want, tol, dtype):
    got = got.to(torch.float64)
    limit = tol + HALF_ULP[dtype] * (want.abs() + tol) + STEP[dtype]
    if dtype == "f16":                   # what does not fit is infinite
        fits = want.abs() + limit < 65504
        got, want, limit = got[fits], want[fits], limit[fits]
    assert bool((got - want).abs().le(limit).all())


def offsets_of(counts, behind=0):
    off = np.concatenate([[0], np.cumsum(counts)])
    return torch.from_numpy(off.astype(np.int32)).cuda(), int(off[-1]) + behind


PRODUCTS = [  # counts, N, H, rows behind
    ([1], 1, 1, 0), ([1], 130, 128, 0), ([0, 3, 0], 7, 50, 2), ([5], 64, 129, 0), ([64, 0, 65, 1], 129, 300, 5), ([63] * 8, 200, 512, 0),
    ([1] * 200, 33, 640, 9), ([128, 129, 0, 127], 128, 256, 0), ([400], 300, 1001, 3), ([700, 0, 1, 900], 257, 384, 0), ([0, 0], 64, 64, 4),
    ([2] * 256, 16, 128, 0), ([300] * 3, 1, 2000, 0), ([1000], 520, 130, 1)]
BIG = [([9000, 0, 8193, 300, 9001, 255, 7000], 1024, 200, 17), ([33000], 1100, 128, 0), ([6000, 5000, 0, 4000, 7100, 1], 1536, 513, 0),
       ([20000, 0, 30001, 20011], 2048, 130, 5)]      # more than the memory-side cache


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("counts,N,H,behind", PRODUCTS + BIG, ids=lambda v: f"{len(v)}x{max(v)}" if isinstance(v, list) else str(v))
def test_product(eqb, dtype, counts, N, H, behind):  # noqa: F811
    say(f"product of {len(counts)} experts, up to {max(counts)} rows, N={N} H={H} {dtype}")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(N * 1000 + H)
    E = len(counts)
    offsets, R = offsets_of(counts, behind)
    x, xs = coded(eqb, rng, R, H)
    w, _ = coded(eqb, rng, E * N, H)
    _, ws = coded(eqb, rng, E * -(-N // BLOCK), H)
    shift = N % 2
    flat = torch.full((R * N + shift,), 7.0, dtype=TYPES[dtype], device="cuda")
    out = flat[shift:].view(R, N)
    e4, e8 = eqb._CODES, eqb._SCALES
    eqb.eqb_experts_product(x.view(e4), xs.view(e8), w.view(E, N, -1).view(e4), ws.view(E, -(-N // BLOCK), -1).view(e8), offsets, out)
    xv = values(x, xs)
    first = 0
    for e, n in enumerate(counts):
        if n:
            s = ws.view(E, -(-N // BLOCK), -1)[e].repeat_interleave(BLOCK, 0)[:N]
            wv = values(w.view(E, N, -1)[e], s)
            p = xv[first:first + n]
            close(out[first:first + n], p @ wv.t(), bound(p, wv, dtype), dtype)
        first += n
    assert bool((out[first:] == 7.0).all())          # rows of no expert
    assert shift == 0 or float(flat[0]) == 7.0


GRADS = [([1], 1, 1), ([0, 0, 5], 7, 50), ([128, 0, 1, 127, 129], 64, 130), ([300, 256, 0], 129, 257), ([0], 33, 64), ([3] * 60, 17, 20),
         ([600, 513], 200, 300), ([1, 0] * 20, 128, 128), ([2000], 300, 100), ([64] * 256, 8, 16)]
BIG_GRADS = [([300, 0, 700, 1, 1300, 129, 128, 900], 1024, 2048), ([2000, 500], 4096, 4096), ([40, 300, 0] * 11, 2048, 2048)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("counts,N,H", GRADS + BIG_GRADS, ids=lambda v: f"{len(v)}x{max(v)}" if isinstance(v, list) else str(v))
def test_grad_weight(eqb, dtype, counts, N, H):  # noqa: F811
    say(f"weight gradient of {len(counts)} experts, up to {max(counts)} rows, N={N} H={H} {dtype}")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(N * 1000 + H + 1)
    E = len(counts)
    offsets, R = offsets_of(counts, 3)
    W = eqb.eqb_column_width(R, E)
    g, gs = coded(eqb, rng, N, W)
    x, xs = coded(eqb, rng, H, W)
    starts, _ = O.columns(R, offsets.cpu().numpy())
    # zeros behind an expert's rows, as the quantization leaves them; what belongs to no block is arbitrary
    for a, n in zip(starts, counts):
        g[:, a + n:a + -(-n // BLOCK) * BLOCK] = 0
    out = torch.full((E, N, H), 7.0, dtype=TYPES[dtype], device="cuda")
    e4, e8 = eqb._CODES, eqb._SCALES
    eqb.eqb_experts_grad_weight(g.view(e4), gs.view(e8), x.view(e4), xs.view(e8), offsets, out)
    gv, xv = values(g, gs), values(x, xs)
    for e, (a, n) in enumerate(zip(starts, counts)):
        m = -(-n // BLOCK) * BLOCK
        if n == 0:
            assert not bool(out[e].any())
            continue
        p, q = gv[:, a:a + m], xv[:, a:a + m]
        close(out[e], p @ q.t(), bound(p, q, dtype), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_numbers_stay_in_their_rows(eqb, dtype):  # noqa: F811
    """A NaN in a row (a column of the weights) makes that row (column) NaN and nothing else."""
    say(f"NaN codes {dtype}")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(5)
    for counts, N, H in (([200, 90], 140, 300), ([20, 9], 140, 300)):
        offsets, R = offsets_of(counts)
        x, xs = coded(eqb, rng, R, H)
        w, _ = coded(eqb, rng, 2 * N, H)
        _, ws = coded(eqb, rng, 2 * 2, H)
        x[5, 130], x[R - 1, 299] = 127, 255
        w[N + 77, 0] = 127                       # expert 1, column 77
        out = torch.zeros((R, N), dtype=TYPES[dtype], device="cuda")
        e4, e8 = eqb._CODES, eqb._SCALES
        eqb.eqb_experts_product(x.view(e4), xs.view(e8), w.view(2, N, -1).view(e4), ws.view(2, 2, -1).view(e8), offsets, out)
        want = torch.zeros((R, N), dtype=torch.bool, device="cuda")
        want[5] = want[R - 1] = True
        want[counts[0]:, 77] = True
        assert bool((out.isnan() == want).all())


def test_scales_of_all_sizes(eqb):  # noqa: F811
    """Powers from 2^-126 to 2^120 whose sums are in range: the instruction's scales and the BF16 path's."""
    say("far scales")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(6)
    offsets, R = offsets_of([150])
    for a, b in ((1, 240), (240, 1), (20, 200), (247, 20), (60, 190)):
        x, xs = coded(eqb, rng, R, 256)
        w, ws = coded(eqb, rng, 130, 256)
        xs.fill_(a)
        ws = torch.full((2, 4), b, dtype=torch.uint8, device="cuda")
        for dtype in ("bf16", "f32"):
            if dtype == "f32" and (min(a, b) < 10 or max(a, b) > 246):
                # codes times 2^-126: below 2^-133 they are lost; 448 2^120 = 1.75 2^128 is no binary32 number, and a
                # scale of 2^120 comes with no such code from one
                continue
            out = torch.zeros((R, 130), dtype=TYPES[dtype], device="cuda")
            e4, e8 = eqb._CODES, eqb._SCALES
            eqb.eqb_experts_product(x.view(e4), xs.view(e8), w.view(1, 130, -1).view(e4), ws.view(1, 2, -1).view(e8), offsets, out)
            p, q = values(x, xs), values(w, ws.repeat_interleave(BLOCK, 0)[:130])
            close(out, p @ q.t(), bound(p, q, dtype), dtype)


def test_offsets_outside_the_rows(eqb):  # noqa: F811
    """Offsets are taken as if they lay within the rows, and a range that ends before it begins is empty."""
    say("offsets outside")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(8)
    R, N, H = 200, 64, 128
    x, xs = coded(eqb, rng, R, H)
    w, _ = coded(eqb, rng, 3 * N, H)
    _, ws = coded(eqb, rng, 3, H)
    e4, e8 = eqb._CODES, eqb._SCALES
    outs = []
    for off in ([0, 70, 200, 200], [-5, 70, 900, 200]):
        out = torch.zeros((R, N), dtype=torch.bfloat16, device="cuda")
        eqb.eqb_experts_product(x.view(e4), xs.view(e8), w.view(3, N, -1).view(e4), ws.view(3, 1, -1).view(e8),
                                torch.tensor(off, dtype=torch.int32, device="cuda"), out)
        outs.append(out)
    assert torch.equal(*outs)


def test_streams_blocks_and_repeats(eqb):  # noqa: F811
    """Capped grids (one block does all tiles), another stream, twice: the same bits, for every tile size."""
    say("products on streams")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(9)
    e4, e8 = eqb._CODES, eqb._SCALES
    for counts, N, H in (([30, 0, 7], 200, 300), ([500, 0, 700, 129], 300, 640), ([9000, 8000, 16000], 1100, 128)):
        E = len(counts)
        offsets, R = offsets_of(counts)
        x, xs = coded(eqb, rng, R, H)
        w, _ = coded(eqb, rng, E * N, H)
        _, ws = coded(eqb, rng, E * -(-N // BLOCK), H)
        W = eqb.eqb_column_width(R, E)
        g, gs = coded(eqb, rng, N, W)
        c, cs = coded(eqb, rng, H, W)

        def calls():
            out = [torch.zeros((R, N), dtype=t, device="cuda") for t in (torch.bfloat16, torch.float32)]
            for o in out:
                eqb.eqb_experts_product(x.view(e4), xs.view(e8), w.view(E, N, -1).view(e4), ws.view(E, -(-N // BLOCK), -1).view(e8), offsets, o)
            out += [torch.empty((E, N, H), dtype=t, device="cuda") for t in (torch.float16, torch.float32)]
            for o in out[2:]:
                eqb.eqb_experts_grad_weight(g.view(e4), gs.view(e8), c.view(e4), cs.view(e8), offsets, o)
            return out

        want = calls()
        s = torch.cuda.Stream()
        for cap in (3, 9, 0):
            eqb.eqb_set_max_blocks(cap)
            try:
                s.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(s):
                    got = calls()
                s.synchronize()
            finally:
                eqb.eqb_set_max_blocks(0)
            for a, b in zip(want, got):
                assert torch.equal(a.view(torch.int16 if a.element_size() == 2 else torch.int32), b.view(torch.int16 if b.element_size() == 2 else torch.int32))
