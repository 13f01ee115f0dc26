"""GPU dispatch and combine with their gradients against the binary64 oracle.

Tolerance.  The plan and the dispatched rows are exact.  A combined value sums K products
in binary32, each product and sum rounded: at most (K + 1) 2^-24 of the sum of the
products' magnitudes, then half an ulp of the row's type (8 significant bits for bf16, so
2^-8 at most; 11 for f16, so 2^-11; none more for f32; below the normal range half of its smallest step).  A
gradient row is one product, rounded.  A gradient of a weight sums H products in any
order: H 2^-24 of the sum of their magnitudes at most."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
STEP = {"f32": 0.0, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def picks(rng, T, K, E, drop=0.0, skew=False):
    if skew:
        idx = np.tile(np.arange(K), (T, 1))
    else:
        idx = np.argsort(rng.random((T, E)), axis=1)[:, :K]
    idx = idx.astype(np.int32)
    idx[rng.random((T, K)) < drop] = -1
    idx[rng.random((T, K)) < drop / 3] = E + 5
    return idx


def plan(eqb, idx, E):  # noqa: F811
    T, K = idx.shape
    off = torch.full((E + 1,), -9, dtype=torch.int32, device="cuda")
    slot = torch.full((T, K), -9, dtype=torch.int32, device="cuda")
    n = eqb.eqb_dispatch_workspace_size(T, K, E)
    ws = torch.full((n,), 0xAB, dtype=torch.uint8, device="cuda") if n else None
    eqb.eqb_dispatch_plan(torch.from_numpy(idx).cuda(), E, off, slot, ws)
    return off, slot


def sorted_plan(idx, E):
    flat = idx.reshape(-1).astype(np.int64)
    inside = np.nonzero((flat >= 0) & (flat < E))[0]
    order = inside[np.argsort(flat[inside], kind="stable")]
    slot = np.full(flat.size, -1)
    slot[order] = np.arange(order.size)
    return np.searchsorted(flat[order], np.arange(E + 1)), slot.reshape(idx.shape)


@pytest.mark.parametrize("T,K,E,drop,skew", [
    (0, 2, 8, 0, False), (1, 1, 8, 0, False), (1, 8, 256, 0, False), (7, 3, 16, 0.3, False), (64, 1, 32, 0, True),
    (1000, 4, 64, 0.1, False), (1024, 4, 128, 0, False), (1025, 4, 128, 0, False), (5000, 7, 8, 0.05, False),
    (4097, 8, 256, 0.02, False), (20000, 16, 32, 0, True), (100003, 5, 64, 0.1, False), (147456, 6, 256, 0, False),
    (3000, 255, 256, 0, False), (600000, 2, 16, 0, True), (50, 2, 8, 1.0, False), (30000, 2, 8, 1.0, True)])
def test_plan(eqb, T, K, E, drop, skew):  # noqa: F811
    say(f"plan T={T} K={K} E={E} drop={drop} skew={skew}")
    idx = picks(np.random.default_rng(T + K), T, K, E, drop, skew)
    off, slot = plan(eqb, idx, E)
    want_off, want_slot = sorted_plan(idx, E) if T * K > 2000 else O.dispatch_plan(idx, E)
    assert np.array_equal(off.cpu().numpy(), want_off)
    assert np.array_equal(slot.cpu().numpy(), want_slot)


def test_plan_with_capped_blocks_and_streams(eqb):  # noqa: F811
    idx = picks(np.random.default_rng(0), 20000, 6, 64, 0.1)
    want = sorted_plan(idx, 64)
    s = torch.cuda.Stream()
    for cap in (1, 3, 0):
        eqb.eqb_set_max_blocks(cap)
        try:
            with torch.cuda.stream(s):
                off, slot = plan(eqb, idx, 64)
                got = off.cpu().numpy(), slot.cpu().numpy()
        finally:
            eqb.eqb_set_max_blocks(0)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


def away(shape, dtype, rng, shift, scale=1.0):
    """Random rows that start `shift` elements past an aligned address."""
    n = int(np.prod(shape))
    flat = torch.empty(n + shift, dtype=dtype, device="cuda")
    t = flat[shift:].view(shape)
    t.copy_(torch.from_numpy(rng.normal(size=shape).astype(np.float32) * scale))
    return t


def f64(t):
    return t.to(torch.float64).cpu().numpy()


SHAPES = [(1, 1, 8, 1, 0), (1, 8, 256, 2048, 0), (2, 2, 16, 3, 1), (5, 3, 32, 7, 0), (33, 4, 8, 8, 0), (65, 5, 64, 16, 1),
          (40, 6, 256, 129, 0), (64, 8, 128, 512, 3), (31, 16, 32, 1000, 0), (19, 2, 8, 1001, 1), (23, 3, 64, 2049, 0),
          (9, 17, 64, 4100, 1), (300, 6, 256, 256, 0), (257, 1, 16, 64, 0), (3, 40, 64, 515, 0), (2, 7, 8, 20000, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,K,E,H,shift", SHAPES)
def test_rows(eqb, dtype, T, K, E, H, shift):  # noqa: F811
    say(f"rows T={T} K={K} E={E} H={H} shift={shift} {dtype}")
    rng = np.random.default_rng(T * 31 + H)
    dt, half, step = TYPES[dtype], HALF_ULP[dtype], STEP[dtype]
    idx = picks(rng, T, K, E, 0.1 if T > 1 else 0.0)
    _, slot = plan(eqb, idx, E)
    s = slot.cpu().numpy()
    R = T * K
    x, rows = away((T, H), dt, rng, shift), away((R, H), dt, rng, shift)
    before = f64(rows)
    eqb.eqb_dispatch(x, slot, rows)
    assert np.array_equal(f64(rows), O.dispatch(f64(x), s, before))

    out, gy = away((R, H), dt, rng, shift), away((T, H), dt, rng, shift)
    weight = torch.from_numpy(rng.random((T, K)).astype(np.float32)).cuda()
    y = away((T, H), dt, rng, shift)
    for w in (weight, None):
        eqb.eqb_combine(out, slot, w, y)
        wn = None if w is None else f64(w)
        want = O.combine(f64(out), s, wn, H)
        size = O.combine(np.abs(f64(out)), s, wn, H)
        assert np.all(np.abs(f64(y) - want) <= (K + 1) * 2.0 ** -24 * size * (1 + half) + half * np.abs(want) + step)

    gr = away((R, H), dt, rng, shift)
    before = f64(gr)
    gw = torch.full((T, K), float("nan"), device="cuda")
    eqb.eqb_combine_backward(gy, out, slot, weight, gr, gw)
    want, wgw = O.combine_backward(f64(gy), f64(out), s, f64(weight), before)
    named = np.zeros(R, dtype=bool)
    named[s[s >= 0]] = True
    assert np.array_equal(f64(gr)[~named], want[~named])
    err = np.abs(f64(gr) - want)[named]
    assert np.all(err <= (half + 2.0 ** -24 * (1 + half)) * np.abs(want[named]) + step)
    _, size = O.combine_backward(np.abs(f64(gy)), np.abs(f64(out)), s, f64(weight), before)
    assert np.all(np.abs(f64(gw) - wgw) <= H * 2.0 ** -24 * size + 1e-44)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropped_pairs_and_short_buffers(eqb, dtype):  # noqa: F811
    """Slots of -1 and slots past the buffer take no part, whatever the rows hold (NaN and infinities included)."""
    rng = np.random.default_rng(8)
    T, K, H, R = 20, 3, 70, 31
    dt = TYPES[dtype]
    s = rng.permutation(T * K).reshape(T, K).astype(np.int32)      # 0 .. 59: 31 and more lie outside
    s[0] = -1
    s[1] = [-5, 2 ** 30, -2 ** 31]
    slot = torch.from_numpy(s).cuda()
    guard = torch.full((R + 40, H), float("nan"), dtype=dt, device="cuda")
    rows = guard[:R]
    rows.copy_(torch.from_numpy(rng.normal(size=(R, H)).astype(np.float32)))
    named = np.zeros(R, dtype=bool)
    named[s[(s >= 0) & (s < R)]] = True
    rows[torch.from_numpy(~named).cuda()] = float("inf")
    x, y = away((T, H), dt, rng, 0), away((T, H), dt, rng, 0)
    weight = torch.from_numpy(rng.random((T, K)).astype(np.float32)).cuda()
    weight[0] = float("nan")
    say(f"dropped pairs {dtype}")
    eqb.eqb_combine(rows, slot, weight, y)
    clean = np.where(named[:, None], np.nan_to_num(f64(rows), posinf=0), 0)
    w = np.nan_to_num(f64(weight))
    half = HALF_ULP[dtype]
    want, size = O.combine(clean, s, w, H), O.combine(np.abs(clean), s, w, H)
    assert np.all(np.abs(f64(y) - want) <= 4 * 2.0 ** -24 * size * (1 + half) + half * np.abs(want) + STEP[dtype])
    assert np.all(f64(y)[0] == 0)
    gr, gw = torch.full((R + 40, H), 7.0, dtype=dt, device="cuda"), torch.full((T, K), 9.0, device="cuda")
    eqb.eqb_combine_backward(x, rows, slot, weight, gr[:R], gw)
    eqb.eqb_dispatch(x, slot, rows)
    assert np.all(f64(gr)[R:] == 7) and np.all(f64(gr)[:R][~named] == 7)
    assert np.all(f64(gw)[(s < 0) | (s >= R)] == 0)
    assert torch.isnan(guard[R:]).all() and torch.isinf(rows[torch.from_numpy(~named).cuda()]).all()
    assert np.array_equal(f64(rows)[named], O.dispatch(f64(x), s, np.zeros((R, H)))[named])


def test_special_values_pass(eqb):  # noqa: F811
    """Infinities and NaN of a named row reach the token's sum and its gradients, and no other token's."""
    T, K, H = 6, 2, 40
    slot = torch.arange(T * K, dtype=torch.int32, device="cuda").view(T, K)
    rows = torch.ones((T * K, H), device="cuda")
    rows[4, 3], rows[7, 5], rows[7, 6] = float("inf"), float("nan"), -float("inf")
    y = torch.empty((T, H), device="cuda")
    w = torch.full((T, K), 0.5, device="cuda")
    eqb.eqb_combine(rows, slot, w, y)
    want = torch.ones((T, H), device="cuda")
    want[2, 3], want[3, 5], want[3, 6] = float("inf"), float("nan"), -float("inf")
    assert torch.equal(torch.nan_to_num(y, nan=77.0), torch.nan_to_num(want, nan=77.0))
    gw = torch.empty((T, K), device="cuda")
    eqb.eqb_combine_backward(torch.ones((T, H), device="cuda"), rows, slot, w, torch.empty_like(rows), gw)
    assert torch.isinf(gw[2, 0]) and torch.isnan(gw[3, 1]) and torch.isfinite(gw).sum() == T * K - 2


def test_rows_past_4_gib(eqb):  # noqa: F811
    """Rows whose byte offsets pass 2^32."""
    R, H, T = 2200000, 2048, 64
    rng = np.random.default_rng(1)
    s = (R - 1 - rng.permutation(T * 2)).reshape(T, 2).astype(np.int32)
    s[:8, 0] = np.arange(8)
    slot = torch.from_numpy(s).cuda()
    say("rows past 4 GiB")
    rows = torch.empty((R, H), dtype=torch.bfloat16, device="cuda")
    x = away((T, H), torch.bfloat16, rng, 0)
    eqb.eqb_dispatch(x, slot, rows)
    at = slot.long()
    assert torch.equal(rows[at[:, 0]], x) and torch.equal(rows[at[:, 1]], x)
    y = torch.empty_like(x)
    eqb.eqb_combine(rows, slot, torch.full((T, 2), 0.5, device="cuda"), y)
    assert torch.equal(y, x)
    gr = torch.empty_like(rows)
    gw = torch.empty((T, 2), device="cuda")
    eqb.eqb_combine_backward(x, rows, slot, torch.ones((T, 2), device="cuda"), gr, gw)
    assert torch.equal(gr[at[:, 1]], x)
    want = (f64(x) ** 2).sum(1)
    assert np.all(np.abs(f64(gw) - want[:, None]) <= H * 2.0 ** -24 * want[:, None])


def test_captured_in_a_graph(eqb):  # noqa: F811
    """Plan, dispatch, combine, balance loss and gradients in one graph, replayed on changing inputs with eager work
    between the replays."""
    T, K, E, H = 3000, 4, 64, 96
    rng = np.random.default_rng(3)
    d = dict(device="cuda")
    idx = torch.zeros((T, K), dtype=torch.int32, **d)
    z = torch.zeros((T, E), dtype=torch.bfloat16, **d)
    x, out = torch.zeros((T, H), dtype=torch.bfloat16, **d), torch.zeros((T * K, H), dtype=torch.bfloat16, **d)
    w = torch.zeros((T, K), **d)

    def buffers():
        return dict(off=torch.zeros(E + 1, dtype=torch.int32, **d), slot=torch.zeros((T, K), dtype=torch.int32, **d),
                    ws=torch.zeros(eqb.eqb_dispatch_workspace_size(T, K, E), dtype=torch.uint8, **d),
                    rows=torch.zeros((T * K, H), dtype=torch.bfloat16, **d), y=torch.zeros((T, H), dtype=torch.bfloat16, **d),
                    gr=torch.zeros((T * K, H), dtype=torch.bfloat16, **d), gw=torch.zeros((T, K), **d),
                    load=torch.zeros((2, E), dtype=torch.int32, **d), tokens=torch.zeros(2, dtype=torch.int32, **d),
                    prob=torch.zeros((2, E), **d), loss=torch.zeros(2, **d), gz=torch.zeros((T, E), **d),
                    bws=torch.zeros(eqb.eqb_balance_workspace_size(E, 2), dtype=torch.uint8, **d))
    gl = torch.ones(2, **d)
    part = eqb.PartOffsets([0, 1000, T])

    def work(b):
        eqb.eqb_dispatch_plan(idx, E, b["off"], b["slot"], b["ws"])
        eqb.eqb_dispatch(x, b["slot"], b["rows"])
        eqb.eqb_combine(out, b["slot"], w, b["y"])
        eqb.eqb_combine_backward(x, out, b["slot"], w, b["gr"], b["gw"])
        eqb.eqb_balance_loss(z.view(torch.int16), idx, K, 0.1, b["load"], b["tokens"], b["prob"], b["loss"], b["bws"],
                             part_off=part)
        eqb.eqb_balance_backward(z.view(torch.int16), b["load"], b["tokens"], K, 0.1, gl, b["gz"], topk_idx=idx,
                                 grad_score=b["gw"], part_off=part)

    a, b = buffers(), buffers()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        work(a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        work(a)
    for r in range(4):
        say(f"graph replay {r}")
        zn = rng.normal(size=(T, E)).astype(np.float32)
        z.copy_(torch.from_numpy(zn))
        idx.copy_(torch.from_numpy(np.argsort(-zn, axis=1)[:, :K].astype(np.int32)))
        for t in (x, out, w):
            t.copy_(torch.from_numpy(rng.normal(size=t.shape).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        work(b)
        torch.cuda.synchronize()
        for k in a:
            if k not in ("ws", "bws"):
                assert torch.equal(a[k], b[k]), (r, k)


def test_capped_blocks(eqb):  # noqa: F811
    """Few blocks walk over all tokens: the same bits as many."""
    rng = np.random.default_rng(5)
    T, K, E, H = 700, 3, 16, 200
    _, slot = plan(eqb, picks(rng, T, K, E, 0.05), E)
    x, out = away((T, H), torch.bfloat16, rng, 0), away((T * K, H), torch.bfloat16, rng, 0)
    w = torch.from_numpy(rng.random((T, K)).astype(np.float32)).cuda()

    def run():
        rows, y = torch.zeros_like(out), torch.zeros_like(x)
        gr, gw = torch.zeros_like(out), torch.zeros((T, K), device="cuda")
        eqb.eqb_dispatch(x, slot, rows)
        eqb.eqb_combine(out, slot, w, y)
        eqb.eqb_combine_backward(x, out, slot, w, gr, gw)
        return rows, y, gr, gw

    want = run()
    for cap in (1, 3, 7):
        say(f"rows, at most {cap} blocks")
        eqb.eqb_set_max_blocks(cap)
        try:
            got = run()
        finally:
            eqb.eqb_set_max_blocks(0)
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_buffers_beyond_the_cache(eqb):  # noqa: F811
    """Rows past 256 MiB take the streamed forms: against torch's own indexing (a combined value within the rounding of
    the products' and sums' order, a weight's gradient within H 2^-24 of its magnitudes)."""
    for T, H, dtype in ((70001, 1024, torch.bfloat16), (40001, 1000, torch.float32), (9001, 8200, torch.float16)):
        K, E = 2, 8
        g = torch.Generator(device="cuda")
        g.manual_seed(T)
        idx = torch.rand((T, E), generator=g, device="cuda").topk(K, dim=1).indices.to(torch.int32)
        _, slot = plan(eqb, idx.cpu().numpy(), E)
        at = slot.long()
        say(f"rows beyond the cache {T} x {H} {dtype}")
        x = torch.randn((T, H), generator=g, device="cuda", dtype=dtype)
        rows = torch.empty((T * K, H), dtype=dtype, device="cuda")
        eqb.eqb_dispatch(x, slot, rows)
        assert all(torch.equal(rows[at[:, k]], x) for k in range(K))
        out = torch.randn((T * K, H), generator=g, device="cuda", dtype=dtype)
        w = torch.rand((T, K), generator=g, device="cuda")
        y = torch.empty_like(x)
        eqb.eqb_combine(out, slot, w, y)
        parts = [w[:, k:k + 1].double() * out[at[:, k]].double() for k in range(K)]
        want, size = parts[0] + parts[1], parts[0].abs() + parts[1].abs()
        half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 0.0}[dtype]
        assert bool(((y.double() - want).abs() <= 3 * 2.0 ** -24 * size * (1 + half) + half * want.abs() + 2.0 ** -25).all())
        gr, gw = torch.empty_like(out), torch.empty_like(w)
        eqb.eqb_combine_backward(x, out, slot, w, gr, gw)
        for k in range(K):
            assert torch.equal(gr[at[:, k]], (w[:, k:k + 1] * x.float()).to(dtype))
            dot, mag = (x.double() * out[at[:, k]].double()), H * 2.0 ** -24
            assert bool(((gw[:, k].double() - dot.sum(1)).abs() <= mag * dot.abs().sum(1)).all())
