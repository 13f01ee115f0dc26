"""GPU codes of rows, dispatched rows, columns and weights, bit for bit against the oracle; the gated activation
within its roundings.

Tolerance of the gate (u = 2^-24): a sigmoid is within 8u (see the routing's test), each product and the fma are
rounded once: 11u of h, 14u of the gradients' magnitudes, then half an ulp of the type (bf16 2^-8, fp16 2^-11 of the value, at
least half its smallest step)."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_experts import HALF_ULP, STEP, TYPES, away, f64, picks, plan

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def values(rng, shape, dtype, kind):
    """Rows of unequal size; zeros; values on codes and on ties; the type's largest, smallest and no numbers."""
    x = rng.normal(size=shape) * np.exp(rng.normal(size=(shape[0],) + (1,) * (len(shape) - 1)) * 2)
    if kind == "ties":
        x = np.round(x * 8) / 8 * np.exp2(rng.integers(-6, 6, size=shape))
    if kind == "odd":
        x[rng.random(shape) < 0.3] = 0
        top = float(torch.finfo(TYPES[dtype]).max)
        flat = x.reshape(-1)
        at = rng.permutation(flat.size)[:max(1, flat.size // 50)]
        flat[at] = rng.choice([top, -top, np.inf, -np.inf, np.nan, 448.0, 449.0, 1e-6, -0.0, float(torch.finfo(TYPES[dtype]).tiny)], size=at.size)
    return x


def placed(x, dtype, shift):
    """x on the GPU, `shift` elements past an aligned address."""
    flat = torch.empty(x.size + shift, dtype=TYPES[dtype], device="cuda")
    t = flat[shift:].view(x.shape)
    t.copy_(torch.from_numpy(x))
    return t


def buffers(eqb, lead, hidden, fill=0xA5):  # noqa: F811
    c = torch.full((*lead, eqb.eqb_code_width(hidden)), fill, dtype=torch.uint8, device="cuda")
    s = torch.full((*lead, eqb.eqb_scale_width(hidden)), fill, dtype=torch.uint8, device="cuda")
    return c.view(eqb._CODES), s.view(eqb._SCALES)


def raw(t):
    return t.view(torch.uint8).cpu().numpy()


def same_codes(got, want):
    """Equal, with any code of no number for any other."""
    nan = (want & 127) == 127
    return np.array_equal(np.where(nan, 127, want), np.where((got & 127) == 127, 127, got))


SIZES = [(1, 1), (1, 128), (3, 7), (5, 129), (4, 511), (7, 512), (2, 513), (33, 1001), (9, 2048), (300, 64), (2, 5000)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,H", SIZES)
def test_rows(eqb, dtype, R, H):  # noqa: F811
    say(f"codes of rows R={R} H={H} {dtype}")
    rng = np.random.default_rng(R * 7 + H)
    for kind in ("normal", "ties", "odd"):
        x = placed(values(rng, (R, H), dtype, kind), dtype, R % 3)
        codes, scales = buffers(eqb, (R,), H)
        eqb.eqb_quantize_rows(x, codes, scales)
        wc, ws = O.quantize_rows(f64(x))
        assert same_codes(raw(codes), wc) and np.array_equal(raw(scales), ws), kind
        # a count on the device: the rows behind it are left as they are
        codes, scales = buffers(eqb, (R,), H)
        for n in (R // 2, -5):
            eqb.eqb_quantize_rows(x, codes, scales, torch.tensor([n], dtype=torch.int32, device="cuda"))
            n = max(0, n)
            if n == R // 2:
                assert same_codes(raw(codes)[:n], wc[:n]) and np.array_equal(raw(scales)[:n], ws[:n])
            assert (raw(codes)[R // 2:] == 0xA5).all() and (raw(scales)[R // 2:] == 0xA5).all()
        eqb.eqb_quantize_rows(x, codes, scales, torch.tensor([R + 9], dtype=torch.int32, device="cuda"))
        assert same_codes(raw(codes), wc)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,K,E,H", [(1, 1, 8, 16), (7, 3, 16, 129), (64, 4, 32, 1000), (33, 8, 256, 2048), (500, 6, 64, 33)])
def test_dispatch(eqb, dtype, T, K, E, H):  # noqa: F811
    say(f"dispatched codes T={T} K={K} E={E} H={H} {dtype}")
    rng = np.random.default_rng(T + H)
    idx = picks(rng, T, K, E, 0.2 if T > 1 else 0.0)
    offsets, slot = plan(eqb, idx, E)
    x = placed(values(rng, (T, H), dtype, "odd"), dtype, 1)
    wc, ws = O.quantize_rows(f64(x))
    codes, scales = buffers(eqb, (T * K,), H)
    eqb.eqb_dispatch_quantized(x, slot, codes, scales)
    s = slot.cpu().numpy()
    seen = np.zeros(T * K, bool)
    for t in range(T):
        for k in range(K):
            if s[t, k] >= 0:
                seen[s[t, k]] = True
                assert same_codes(raw(codes)[s[t, k]], wc[t]) and np.array_equal(raw(scales)[s[t, k]], ws[t])
    assert (raw(codes)[~seen] == 0xA5).all() and (raw(scales)[~seen] == 0xA5).all()
    # fewer rows than slots name: the others are dropped
    codes, scales = buffers(eqb, (max(1, T * K // 2),), H)
    eqb.eqb_dispatch_quantized(x, slot, codes, scales)


COUNTS = [[1], [0, 0, 5], [128, 0, 1, 127, 129], [300, 256, 0, 0, 64], [0], [3] * 40, [1, 0] * 128, [700]]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: f"{len(c)}x{max(c)}")
def test_columns(eqb, dtype, counts):  # noqa: F811
    rng = np.random.default_rng(sum(counts) + len(counts))
    for H, behind in ((1, 0), (130, 7), (200, 260)):
        R = sum(counts) + behind
        if R == 0:
            continue
        say(f"codes of columns {len(counts)} experts, {R} rows of {H} {dtype}")
        x = placed(values(rng, (R, H), dtype, "odd" if H == 130 else "normal"), dtype, H % 2)
        offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        W = eqb.eqb_column_width(R, len(counts))
        assert W == O.columns(R, offsets)[1]
        codes, scales = buffers(eqb, (H,), W)
        wc, ws = O.quantize_columns(f64(x), offsets, raw(codes).copy(), raw(scales).copy())
        eqb.eqb_quantize_columns(x, torch.from_numpy(offsets).cuda(), codes, scales)
        assert same_codes(raw(codes), wc) and np.array_equal(raw(scales), ws)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("E,N,H", [(1, 1, 1), (3, 128, 128), (2, 129, 127), (8, 7, 300), (5, 260, 520), (256, 2, 130), (2, 640, 64)])
def test_weights(eqb, dtype, E, N, H):  # noqa: F811
    say(f"codes of weights E={E} N={N} H={H} {dtype}")
    rng = np.random.default_rng(E + N + H)
    w = placed(values(rng, (E, N, H), dtype, "odd" if E == 5 else "ties"), dtype, 1)
    up = lambda n: -(-n // 128)  # noqa: E731
    codes, _ = buffers(eqb, (E, N), H)
    _, scales = buffers(eqb, (E, up(N)), H)
    codes_t, _ = buffers(eqb, (E, H), N)
    _, scales_t = buffers(eqb, (E, up(H)), N)
    eqb.eqb_quantize_weights(w, codes, scales, codes_t, scales_t)
    w64 = f64(w)
    for c, s, v in ((codes, scales, w64), (codes_t, scales_t, w64.transpose(0, 2, 1).copy())):
        wc, ws = O.quantize_weights(v)
        assert same_codes(raw(c), wc) and np.array_equal(raw(s), ws)
    both = raw(codes).copy(), raw(scales_t).copy(), raw(codes_t).copy()
    # one way only: the other is not touched
    for t in (codes, scales, codes_t, scales_t):
        t.view(torch.uint8).fill_(0xA5)
    eqb.eqb_quantize_weights(w, codes, scales)
    assert np.array_equal(raw(codes), both[0]) and (raw(codes_t) == 0xA5).all() and (raw(scales_t) == 0xA5).all()
    codes.view(torch.uint8).fill_(0xA5)
    eqb.eqb_quantize_weights(w, codes_t=codes_t, scales_t=scales_t)
    assert np.array_equal(raw(codes_t), both[2]) and np.array_equal(raw(scales_t), both[1]) and (raw(codes) == 0xA5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("R,F", [(1, 1), (3, 8), (5, 130), (64, 512), (7, 1001), (200, 33), (2, 3001)])
def test_gate(eqb, dtype, R, F):  # noqa: F811
    say(f"gate R={R} F={F} {dtype}")
    rng = np.random.default_rng(R + F)
    dt, half, step = TYPES[dtype], HALF_ULP[dtype], STEP[dtype]
    x = away((R, 2 * F), dt, rng, F % 2, 3.0)
    gh = away((R, F), dt, rng, F % 2)
    h, gx = away((R, F), dt, rng, 1), away((R, 2 * F), dt, rng, 1)
    h0, gx0 = f64(h), f64(gx)
    n = R - R // 3
    count = torch.tensor([n], dtype=torch.int32, device="cuda")
    eqb.eqb_gated(x, h, count)
    want = O.gated(f64(x))
    tol = (11 * U + half) * np.abs(want) + step + 2.0 ** -140
    assert (np.abs(f64(h) - want) <= tol)[:n].all() and np.array_equal(f64(h)[n:], h0[n:])
    eqb.eqb_gated_backward(gh, x, gx, count)
    want, size = O.gated_backward(f64(gh), f64(x))
    tol = 14 * U * size + half * np.abs(want) * (1 + 14 * U) + step + 2.0 ** -140
    # the rounding is of the computed value
    tol += half * 14 * U * size
    assert (np.abs(f64(gx) - want) <= tol)[:n].all() and np.array_equal(f64(gx)[n:], gx0[n:])
    # as codes: of values within 11u, so each is the code of a value that near
    codes, scales = buffers(eqb, (R,), F)
    eqb.eqb_gated_quantize(x, codes, scales, count)
    v = O.decode(raw(codes), raw(scales))[:n, :F]
    exact = O.gated(f64(x))[:n]
    power = np.repeat(np.exp2(raw(scales).astype(float) - 127), 128, 1)[:n, :F]
    assert (np.abs(v - exact) <= (2.0 ** -4 + 12 * U) * np.abs(exact) + power * 2.0 ** -10 * (1 + U)).all()
    top = np.zeros_like(exact)
    for j in range(0, F, 128):
        top[:, j:j + 128] = np.abs(exact[:, j:j + 128]).max(1, keepdims=True)
    assert (top <= 448 * power * (1 + 12 * U)).all() and ((top > 224 * power * (1 - 12 * U)) | (power == 2.0 ** -126)).all()
    assert (raw(codes)[n:] == 0xA5).all() and (raw(scales)[n:] == 0xA5).all() and not raw(codes)[:n, F:].any()


def test_gate_of_large_and_odd_values(eqb):  # noqa: F811
    """Far gates (the sigmoid's ends), zeros, and values that are no numbers stay where they are."""
    say("gate of odd values")
    g = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 88.0, -88.0, 105.0, -105.0, 1e4, -1e4, 3e38, -3e38, float("nan"), 5.0], device="cuda")
    u = torch.full_like(g, 2.0)
    u[13] = float("nan")
    x = torch.cat([g, u])[None]
    h, gx = torch.empty((1, 14), device="cuda"), torch.empty((1, 28), device="cuda")
    eqb.eqb_gated(x, h)
    eqb.eqb_gated_backward(torch.ones((1, 14), device="cuda"), x, gx)
    want, (grad, size) = O.gated(f64(x)), O.gated_backward(np.ones((1, 14)), f64(x))
    assert np.isnan(f64(h)[0, 12:]).all() and np.isnan(f64(gx)[0, [12, 13]]).all()
    for got, w, m in ((f64(h)[0, :12], want[0, :12], np.abs(want[0, :12])), (f64(gx)[0, :12], grad[0, :12], size[0, :12]),
                      (f64(gx)[0, 14:26], grad[0, 14:26], size[0, 14:26])):
        with np.errstate(over="ignore"):
            big = np.abs(w) > 3.4e38
        assert np.isinf(got[big]).all()
        # e^-88 is no normal number: it may count as 0, and so may what it is multiplied with up to 1e4
        assert (np.abs(got - w)[~big] <= 14 * U * m[~big] + 1e4 * 2.0 ** -125).all()


def test_streams_and_blocks(eqb):  # noqa: F811
    """Every call on a stream of its own and with capped grids: the same bits."""
    say("codes on streams")
    rng = np.random.default_rng(0)
    x = away((700, 2 * 640), torch.bfloat16, rng, 0)
    offsets = torch.tensor([0, 130, 130, 700], dtype=torch.int32, device="cuda")
    slot = torch.randperm(700, device="cuda", dtype=torch.int64).to(torch.int32).view(350, 2)

    def calls():
        out = []
        c = buffers(eqb, (700,), 1280)
        eqb.eqb_quantize_rows(x, *c)
        out += c
        c = buffers(eqb, (700,), 1280)
        eqb.eqb_dispatch_quantized(x[:350], slot, *c)
        out += c
        c = buffers(eqb, (1280,), eqb.eqb_column_width(700, 3))
        eqb.eqb_quantize_columns(x, offsets, *c)
        out += c
        c = buffers(eqb, (700,), 640)
        eqb.eqb_gated_quantize(x, *c)
        out += c
        h, gx = torch.empty((700, 640), dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
        eqb.eqb_gated(x, h)
        eqb.eqb_gated_backward(h, x, gx)
        return out + [h, gx]

    want = calls()
    s = torch.cuda.Stream()
    for cap in (1, 5, 0):
        eqb.eqb_set_max_blocks(cap)
        try:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got = calls()
            s.synchronize()
        finally:
            eqb.eqb_set_max_blocks(0)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(want, got))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("low", [False, True])
def test_gated_codes_are_the_exact_products(eqb, dtype, low):  # noqa: F811
    """Bit for bit the codes of the products in 64 bits, of ordinary gates and of gates whose sigmoid has few bits or
    none in 32 (2^-52 to 2^-126 there: the products of 37 bits leave one code in 2^32 open, and none of these)."""
    say(f"exact gated codes {dtype} low={low}")
    rng = np.random.default_rng(40 + low)
    R, F = 300, 1000
    g = rng.uniform(-94, -82, size=(R, 1)) + rng.uniform(-3, 3, size=(R, F)) if low else rng.normal(size=(R, F)) * 3
    u = rng.normal(size=(R, F)) * (np.exp2(rng.integers(2, 9, size=(R, F))) if low else 1.0)
    x = torch.from_numpy(np.concatenate([g, u], 1)).to(TYPES[dtype]).cuda()
    codes, scales = buffers(eqb, (R,), F)
    eqb.eqb_gated_quantize(x, codes, scales)
    wc, ws = O.quantize_rows(O.gated(f64(x)))
    assert (wc[:, :F] & 127 != 0).mean() > 0.5
    assert same_codes(raw(codes), wc) and np.array_equal(raw(scales), ws)


def test_columns_of_descending_offsets(eqb):  # noqa: F811
    """Offsets that do not ascend name no rows: nothing is read or written before or behind the rows."""
    say("columns of descending offsets")
    R, H = 400, 70
    around = torch.full((3 * R, H), 3.0, device="cuda")
    x = around[R:2 * R].fill_(1.0)
    for off in ([0, 390, 130, 400], [400, 0, 400, 0], [300, 300, 10, 10], [-5, 900, 200, -1]):
        codes, scales = buffers(eqb, (H + 1,), eqb.eqb_column_width(R, 3))
        eqb.eqb_quantize_columns(x, torch.tensor(off, dtype=torch.int32, device="cuda"), codes[:-1], scales[:-1])
        # the fill, zeros, and 1 = 256 2^-8
        assert np.isin(raw(codes), [0xA5, 0, 0x78]).all() and np.isin(raw(scales), [0xA5, 119]).all()
        assert (raw(codes)[-1] == 0xA5).all() and (raw(scales)[-1] == 0xA5).all()


def test_more_than_the_cache_holds(eqb):  # noqa: F811
    """Calls over more than 256 MiB, which pass the caches by: the bits of the same rows in calls of a quarter (and of
    columns the transposed rows')."""
    say("codes of large tensors")
    rng = torch.Generator(device="cuda")
    rng.manual_seed(3)
    R, H = 66048, 2048
    x = torch.randn((R, H), generator=rng, device="cuda", dtype=torch.bfloat16)
    quarters = [slice(i * R // 4, (i + 1) * R // 4) for i in range(4)]
    same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))  # noqa: E731

    say("rows and dispatch")
    c, s = buffers(eqb, (R,), H)
    eqb.eqb_quantize_rows(x, c, s)
    for q in quarters:
        qc, qs = buffers(eqb, (R // 4,), H)
        eqb.eqb_quantize_rows(x[q], qc, qs)
        assert same(c[q], qc) and same(s[q], qs)
    slot = torch.randperm(2 * R, generator=rng, device="cuda").to(torch.int32).view(R, 2)
    dc, ds = buffers(eqb, (2 * R,), H)
    eqb.eqb_dispatch_quantized(x, slot, dc, ds)
    token = torch.empty(2 * R, dtype=torch.int64, device="cuda")
    token[slot.view(-1).long()] = torch.arange(R, device="cuda").repeat_interleave(2)
    assert torch.equal(dc.view(torch.uint8), c.view(torch.uint8)[token]) and torch.equal(ds.view(torch.uint8), s.view(torch.uint8)[token])
    del dc, ds, token

    say("columns")
    W = eqb.eqb_column_width(R, 1)
    cc, cs = buffers(eqb, (H,), W)
    eqb.eqb_quantize_columns(x, torch.tensor([0, R], dtype=torch.int32, device="cuda"), cc, cs)
    tc, ts = buffers(eqb, (H,), R)
    eqb.eqb_quantize_rows(x.t().contiguous(), tc, ts)
    assert same(cc[:, :R].contiguous(), tc) and torch.equal(cs.view(torch.uint8)[:, :R // 128], ts.view(torch.uint8)[:, :R // 128])

    say("weights")
    E = 36
    w = torch.randn((E, 2048, 2048), generator=rng, device="cuda", dtype=torch.bfloat16)
    whole = [*buffers(eqb, (E, 2048), 2048), *buffers(eqb, (E, 2048), 2048)]
    whole[1::2] = [buffers(eqb, (E, 16), 2048)[1] for _ in range(2)]
    eqb.eqb_quantize_weights(w, *whole)
    for e in range(0, E, 9):
        part = [t[e:e + 9].clone().view(torch.uint8).fill_(1).view(t.dtype) for t in whole]
        eqb.eqb_quantize_weights(w[e:e + 9], *part)
        assert all(same(a[e:e + 9], b) for a, b in zip(whole, part))
    del w, whole, part

    say("gates")
    g = torch.randn((R, 2 * H), generator=rng, device="cuda", dtype=torch.bfloat16)
    h, gx = torch.empty_like(x), torch.empty_like(g)
    c, s = buffers(eqb, (R,), H)
    eqb.eqb_gated(g, h)
    eqb.eqb_gated_backward(x, g, gx)
    eqb.eqb_gated_quantize(g, c, s)
    for q in quarters:
        qh, qg, (qc, qs) = torch.empty_like(x[q]), torch.empty_like(g[q]), buffers(eqb, (R // 4,), H)
        eqb.eqb_gated(g[q], qh)
        eqb.eqb_gated_backward(x[q], g[q], qg)
        eqb.eqb_gated_quantize(g[q], qc, qs)
        assert same(h[q], qh) and same(gx[q], qg) and same(c[q], qc) and same(s[q], qs)
