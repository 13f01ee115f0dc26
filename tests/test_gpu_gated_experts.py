"""The operators together, as a layer uses them: routing by scores, the plan, the experts in 8 bits, the combine
and all gradients; the handles on streams of their own, captured in a graph, with dropped pairs and empty batches.

Each step's result is compared with the oracle's on what that step was given, so that an earlier step's rounding
does not enter; the products' tolerance is that of their own test."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from oracle import train_oracle as T
from paper_2609_28053_amd import ExpertRows, GatedExperts, ScoredRouter, eqb
from test_gpu_balance import say
from test_gpu_codes import raw
from test_gpu_experts import TYPES, f64
from test_gpu_products import bound, close
from test_gpu_train_handles import busy

pytestmark = pytest.mark.gpu
D = dict(device="cuda")


def layer(seed, T_, E, K, H, F, dtype="bf16"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = TYPES[dtype]
    new = lambda *s, scale=1.0: (torch.randn(s, generator=g, **D) * scale).to(dt)  # noqa: E731
    return dict(x=new(T_, H), up=new(E, 2 * F, H, scale=H ** -0.5), down=new(E, H, F, scale=F ** -0.5),
                z=new(T_, E), bias=torch.randn(E, generator=g, **D) * 0.1, grad_y=new(T_, H))


def one_pass(router, rows, experts, i, stream=None):
    idx, weight = router.forward(i["z"], stream=stream)
    rows.plan(idx, stream=stream)
    out, saved = experts.forward(i["x"], rows, stream=stream)
    y = rows.combine(out, weight, stream=stream)
    grad_out, grad_weight = rows.combine_backward(i["grad_y"], out, weight, stream=stream)
    grad_rows, grad_up, grad_down = experts.backward(grad_out, saved, stream=stream)
    grad_x = rows.combine(grad_rows, stream=stream)
    grad_z = router.backward(i["z"], idx, grad_weight, stream=stream)
    return dict(idx=idx, weight=weight, out=out, y=y, grad_weight=grad_weight, grad_up=grad_up, grad_down=grad_down,
                grad_x=grad_x, grad_z=grad_z, offsets=rows.offsets, slot=rows.slot, saved=saved, grad_out=grad_out)


def T_of(i):
    return i["x"].shape[0]


KEYS = ("idx", "weight", "y", "grad_weight", "grad_up", "grad_down", "grad_x", "grad_z")


def made(i, K, **more):
    E = i["up"].shape[0]
    return (ScoredRouter(E, K, i["bias"], **more), ExpertRows(T_of(i), E, K), GatedExperts(i["up"], i["down"]))


@pytest.mark.parametrize("T_,E,K,H,F,dtype,more", [
    (1, 8, 2, 64, 32, "bf16", {}), (300, 16, 4, 200, 130, "bf16", dict(groups=4, top_groups=2, group_top=2)),
    (257, 32, 3, 129, 65, "f16", dict(score="softmax", normalize=False)), (500, 8, 2, 128, 256, "f32", dict(scale=2.5))])
def test_a_layer(T_, E, K, H, F, dtype, more):
    say(f"a layer T={T_} E={E} K={K} H={H} F={F} {dtype}")
    i = layer(T_ + E, T_, E, K, H, F, dtype)
    if T_ > 200:
        i["z"][5, 1:] = -np.inf          # one expert is left
        i["z"][7] = -np.inf              # none
    router, rows, experts = made(i, K, **more)
    got = one_pass(router, rows, experts, i)
    z = f64(i["z"])
    idx, weight = O.route(z, i["bias"].cpu().numpy(), K, more.get("score") == "softmax", more.get("groups", 1), more.get("top_groups", 1),
                          more.get("group_top", 1), more.get("normalize", True), more.get("scale", 1.0))
    assert np.array_equal(got["idx"].cpu().numpy(), idx) and np.allclose(got["weight"].cpu().numpy(), weight, rtol=2e-5, atol=1e-30)
    off, slot = T.dispatch_plan(idx, E)
    assert np.array_equal(got["offsets"].cpu().numpy(), off) and np.array_equal(got["slot"].cpu().numpy(), slot)
    n = int(off[-1])
    x, gate, _, _ = got["saved"]
    c = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()  # noqa: E731

    def product(rows64, w64, result, transposed):
        """The experts' rows (binary64 [n,.]) through the codes of w64 [E,N,H]."""
        pc, ps = O.quantize_rows(rows64)
        p = c(O.decode(pc, ps))
        wc, ws = O.quantize_weights(w64.transpose(0, 2, 1).copy() if transposed else w64)
        w = c(O.decode_weights(wc, ws))
        for e in range(E):
            a, b = int(off[e]), int(off[e + 1])
            if b > a:
                close(result[a:b], p[a:b] @ w[e].t(), bound(p[a:b], w[e], dtype), dtype)

    def gradient(g64, x64, result):
        """grad[e] from the columns' codes of what each expert's rows were."""
        W = O.columns(g64.shape[0], off)[1]
        new = lambda w: (np.zeros((w, W), np.uint8), np.zeros((w, -(-W // 512) * 4), np.uint8))  # noqa: E731
        g = c(O.decode(*O.quantize_columns(g64, off, *new(g64.shape[1]))))
        v = c(O.decode(*O.quantize_columns(x64, off, *new(x64.shape[1]))))
        starts = O.columns(g64.shape[0], off)[0]
        for e in range(E):
            a, m = starts[e], -(-int(off[e + 1] - off[e]) // 128) * 128
            p, q = g[:, a:a + m], v[:, a:a + m]
            close(result[e], p @ q.t(), bound(p, q, "f32") if m else torch.zeros_like(result[e], dtype=torch.float64), "f32")

    rows64 = np.zeros((T_ * K, H))
    for t in range(T_):
        for k in range(K):
            if slot[t, k] >= 0:
                rows64[slot[t, k]] = f64(x)[t]
    product(rows64[:n], f64(i["up"]), gate, False)
    # the second product takes the codes of the gate's values in binary32: compared through them
    codes, scales = experts._codes(T_ * K, F, "cuda")
    eqb.eqb_gated_quantize(gate, codes, scales, got["offsets"][E:])
    v = O.decode(raw(codes), raw(scales))[:n, :F]
    assert np.allclose(v, O.gated(f64(gate)[:n]), rtol=2.0 ** -4 + 1e-6, atol=np.abs(v).max() * 2.0 ** -17 if n else 0)
    product(v, f64(i["down"]), got["out"], False)
    # backward, each step from what it was given
    gout = f64(got["grad_out"])[:n]
    hidden = torch.empty((T_ * K, F), dtype=TYPES[dtype], **D)
    eqb.eqb_gated(gate, hidden, got["offsets"][E:])
    gradient(gout, f64(hidden)[:n], got["grad_down"])
    again = GatedExperts(i["up"], i["down"])
    grad_hidden = again._product((lambda q: (eqb.eqb_quantize_rows(got["grad_out"], *q, got["offsets"][E:]), q)[1])(again._codes(T_ * K, H, "cuda")),
                                 again.down, True, got["offsets"], F, TYPES[dtype])
    product(gout, f64(i["down"]), grad_hidden, True)
    grad_gate = torch.empty_like(gate)
    eqb.eqb_gated_backward(grad_hidden, gate, grad_gate, got["offsets"][E:])
    gradient(f64(grad_gate)[:n], rows64[:n], got["grad_up"])
    # the tokens' gradient: the rows' product, summed over K
    grad_rows, _, _ = experts.backward(got["grad_out"], got["saved"])
    product(f64(grad_gate)[:n], f64(i["up"]), grad_rows, True)
    assert torch.equal(rows.combine(grad_rows, slot=got["slot"]), got["grad_x"])
    grad, size = O.route_backward(z, idx, f64(got["grad_weight"]), more.get("score") == "softmax", more.get("normalize", True), more.get("scale", 1.0))
    assert (np.abs(got["grad_z"].cpu().numpy() - grad) <= 2e-5 * size + 1e-30).all()


def test_gradients_are_the_differences():
    """A layer whose values are all codes (small integers in every block), so that quantization changes nothing: the whole
    pass against differences of the same layer in binary64.  Rounding of results to binary32 and second-order terms of a
    step of 2^-10: 1e-4 of the gradients' size is more than both."""
    say("differences")
    rng = np.random.default_rng(1)
    T_, E, K, H, F = 6, 8, 2, 8, 4
    x = rng.integers(-3, 4, size=(T_, H)).astype(np.float64)
    up, down = rng.integers(-1, 2, size=(E, 2 * F, H)) * 0.5, rng.integers(-2, 3, size=(E, H, F)) * 0.25
    z, gy = rng.normal(size=(T_, E)), rng.integers(-2, 3, size=(T_, H)).astype(np.float64)
    t = lambda v: torch.from_numpy(np.ascontiguousarray(v)).to(torch.float32).cuda()  # noqa: E731
    router, rows, experts = ScoredRouter(E, K), ExpertRows(T_, E, K), GatedExperts(t(up), t(down))
    idx, weight = router.forward(t(z))
    rows.plan(idx)
    out, saved = experts.forward(t(x), rows)
    _, grad_weight = rows.combine_backward(t(gy), out, weight)
    grad_z = router.backward(t(z), idx, grad_weight)
    ii = idx.cpu().numpy()

    def y_of(z, codes):
        s = O.scores(z, False)
        total = 0.0
        for tt in range(T_):
            w = s[tt, ii[tt]] / s[tt, ii[tt]].sum()
            for k in range(K):
                a = up[ii[tt, k]] @ x[tt]
                h = O.gated(a[None])
                if codes:                        # the rows' codes that the second product takes
                    h = O.decode(*O.quantize_rows(h))[:, :F]
                total += w[k] * (down[ii[tt, k]] @ h[0]) @ gy[tt]
        return total

    h = 2.0 ** -10
    for tt in range(T_):
        for e in range(E):
            d = np.zeros_like(z)
            d[tt, e] = h
            want = (y_of(z + d, True) - y_of(z - d, True)) / (2 * h)
            assert abs(float(grad_z[tt, e]) - want) <= 1e-4 * (1 + abs(want)) + 1e-4 * float(np.abs(gy[tt]).sum())


def test_streams_and_reuse():
    """stream= behind a busy stream with inputs dropped meanwhile: the same bits as on the current stream."""
    say("gated experts on a stream")
    i = layer(3, 600, 16, 4, 256, 192)
    want = {k: v.clone() for k, v in one_pass(*made(i, 4), i).items() if k in KEYS}
    torch.cuda.synchronize()
    i, handles = layer(3, 600, 16, 4, 256, 192), None
    handles = made(i, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    busy(s)
    got = one_pass(*handles, i, stream=s)
    sizes = [(t.shape, t.dtype) for t in i.values()]
    del i, handles
    got = {k: got[k] for k in KEYS}
    junk = [torch.empty(shape, dtype=dtype, **D).view(torch.uint8).fill_(0xFF) for shape, dtype in sizes for _ in range(2)]
    s.synchronize()
    torch.cuda.synchronize()
    assert len(junk) and all(torch.equal(want[k], got[k]) for k in KEYS)


def test_captured_and_replayed():
    """Two graphs of the same handles, replayed in turn with eager passes between: every replay is the eager result."""
    say("gated experts captured")
    T_, E, K, H, F = 400, 16, 3, 192, 130
    router, rows, experts = made(layer(0, T_, E, K, H, F), K)
    graphs = []
    for seed in (1, 2):
        i = layer(seed, T_, E, K, H, F)
        i["bias"] = router.bias
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            one_pass(router, rows, experts, i)
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = one_pass(router, rows, experts, i)
        graphs.append((g, i, out))
    for turn in range(4):
        for seed, (g, i, out) in enumerate(graphs):
            fresh = layer(10 * turn + seed, T_, E, K, H, F)
            for k in ("x", "z", "grad_y"):
                i[k].copy_(fresh[k])
            g.replay()
            torch.cuda.synchronize()
            got = {k: out[k].clone() for k in KEYS}
            want = one_pass(router, rows, experts, i)
            torch.cuda.synchronize()
            assert all(torch.equal(want[k], got[k]) for k in KEYS), (turn, seed)


def test_an_empty_batch_and_no_pairs():
    say("empty batches")
    i = layer(4, 0, 8, 2, 64, 48)
    router, rows, experts = made(i, 2)
    got = one_pass(router, rows, experts, i)
    assert not got["grad_up"].any() and not got["grad_down"].any() and got["y"].shape == (0, 64)
    i = layer(5, 40, 8, 2, 64, 48)
    i["z"].fill_(-np.inf)
    router, rows, experts = made(i, 2)
    got = one_pass(router, rows, experts, i)
    assert bool((got["idx"] == -1).all()) and not got["y"].any() and not got["grad_up"].any() and not got["grad_x"].any() and not got["grad_z"].any()


def test_refresh_takes_new_weights():
    say("new weights")
    i, j = layer(6, 100, 8, 2, 64, 48), layer(7, 100, 8, 2, 64, 48)
    router, rows, experts = made(i, 2)
    first = one_pass(router, rows, experts, i)
    experts.refresh(j["up"], j["down"])
    second = one_pass(router, rows, experts, i)
    assert not torch.equal(first["y"], second["y"])
    fresh = one_pass(router, ExpertRows(100, 8, 2), GatedExperts(j["up"], j["down"]), i)
    assert all(torch.equal(second[k], fresh[k]) for k in KEYS)
    with pytest.raises(ValueError):
        experts.refresh(j["up"][:4], j["down"])
    # serving keeps nothing for a backward pass
    out, saved = experts.forward(i["x"], rows, train=False)
    assert saved is None and torch.equal(rows.combine(out, second["weight"]), second["y"])
