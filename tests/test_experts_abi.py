"""The C ABI of the routing by scores and of the 8-bit products without a GPU: every wrong argument is
refused before the HIP runtime is touched, and the binding and the handles refuse what they can see."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.environ.get("EQB_LIB", os.path.join(ROOT, "paper_2609_28053_amd", "libeqb.so"))
OK, INVALID, UNSUPPORTED = 0, 1, 2
V, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
FAKE = V(0x10000)       # never dereferenced: the calls below fail their checks first
ODD1, ODD2, ODD8 = V(0x10001), V(0x10002), V(0x10008)
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    lib = ctypes.CDLL(LIB)
    lib.eqb_route_scored.argtypes = [V, V, i64] + [i32] * 7 + [f64, i32, V, V, V]
    lib.eqb_route_scored_backward.argtypes = [V, V, V, i64] + [i32] * 4 + [f64, i32, V, V]
    for name, args in (("code_width", [i64]), ("scale_width", [i64]), ("column_width", [i64, i32])):
        getattr(lib, "eqb_" + name).argtypes = args
        getattr(lib, "eqb_" + name).restype = i64
    lib.eqb_quantize_rows.argtypes = [V, V, i64, i32, i32, V, V, V]
    lib.eqb_dispatch_quantized.argtypes = [V, V, i64, i32, i64, i32, i32, V, V, V]
    lib.eqb_quantize_columns.argtypes = [V, V, i64, i32, i32, i32, V, V, V]
    lib.eqb_quantize_weights.argtypes = [V, i32, i32, i32, i32, V, V, V, V, V]
    lib.eqb_experts_product.argtypes = [V] * 5 + [i64, i32, i32, i32, i32, V, V]
    lib.eqb_experts_grad_weight.argtypes = [V] * 5 + [i64, i32, i32, i32, i32, V, V]
    lib.eqb_gated.argtypes = [V, V, i64, i32, i32, V, V]
    lib.eqb_gated_quantize.argtypes = [V, V, i64, i32, i32, V, V, V]
    lib.eqb_gated_backward.argtypes = [V, V, V, i64, i32, i32, V, V]
    return lib


def test_route_scored_refuses(lib):
    def call(z=FAKE, b=FAKE, T=64, E=16, K=2, g=4, tg=2, gt=2, score=0, norm=1, scale=1.0, dt=1, idx=FAKE, w=FAKE):
        return lib.eqb_route_scored(z, b, T, E, K, g, tg, gt, score, norm, scale, dt, idx, w, None)

    assert call(T=-1) == call(T=1 << 31) == call(T=1 << 30) == call(K=0) == call(K=16) == INVALID
    assert call(E=12) == call(E=512) == call(E=4) == UNSUPPORTED
    assert call(g=0) == call(g=3) == call(g=32) == call(tg=0) == call(tg=5) == call(gt=0) == call(gt=3) == INVALID
    assert call(g=16, tg=16) == call(K=9) == INVALID                 # groups of one have no second; two groups of four hold eight
    assert call(score=2) == call(dt=3) == call(dt=-1) == call(scale=NAN) == call(scale=INF) == call(scale=1e300) == INVALID
    assert call(z=None) == call(idx=None) == call(w=None) == INVALID
    assert call(z=ODD8) == call(b=ODD2) == call(idx=ODD1) == call(w=ODD2) == UNSUPPORTED
    assert call(T=0) == call(T=0, z=None, b=None, idx=None, w=None) == OK


def test_route_scored_backward_refuses(lib):
    def call(z=FAKE, idx=FAKE, g=FAKE, T=64, E=16, K=2, score=0, norm=1, scale=1.0, dt=1, gz=FAKE):
        return lib.eqb_route_scored_backward(z, idx, g, T, E, K, score, norm, scale, dt, gz, None)

    assert call(T=-1) == call(T=1 << 30) == call(K=0) == call(K=16) == call(score=-1) == call(dt=3) == call(scale=NAN) == INVALID
    assert call(E=7) == UNSUPPORTED
    assert call(z=None) == call(idx=None) == call(g=None) == call(gz=None) == INVALID
    assert call(z=ODD8) == call(gz=ODD8) == call(idx=ODD2) == call(g=ODD1) == UNSUPPORTED
    assert call(T=0, z=None) == OK


def test_widths(lib):
    from paper_2609_28053_amd import eqb
    for h in (-3, 0, 1, 127, 128, 129, 512, 513, 1001, 4096, 1 << 24):
        assert lib.eqb_code_width(h) == eqb.eqb_code_width(h) == (0 if h < 1 else -(-h // 128) * 128)
        assert lib.eqb_scale_width(h) == eqb.eqb_scale_width(h) == (0 if h < 1 else -(-(-(-h // 128)) // 4) * 4)
        for E in (0, 1, 7, 256, 257):
            want = 0 if h < 0 or not 1 <= E <= 256 else 128 * (h // 128 + E)
            assert lib.eqb_column_width(h, E) == eqb.eqb_column_width(h, E) == want


def test_codes_refuse(lib):
    def rows(x=FAKE, count=None, R=8, H=64, dt=1, c=FAKE, s=FAKE):
        return lib.eqb_quantize_rows(x, count, R, H, dt, c, s, None)

    def gated(x=FAKE, count=None, R=8, H=64, dt=1, c=FAKE, s=FAKE):
        return lib.eqb_gated_quantize(x, count, R, H, dt, c, s, None)

    def dispatch(x=FAKE, slot=FAKE, T=4, K=2, R=8, H=64, dt=1, c=FAKE, s=FAKE):
        return lib.eqb_dispatch_quantized(x, slot, T, K, R, H, dt, c, s, None)

    def columns(x=FAKE, off=FAKE, R=8, E=3, H=64, dt=1, c=FAKE, s=FAKE):
        return lib.eqb_quantize_columns(x, off, R, E, H, dt, c, s, None)

    for f in (rows, gated, dispatch, columns):
        assert f(R=-1) == f(R=1 << 31) == f(H=0) == f(H=(1 << 24) + 1) == f(dt=3) == f(dt=-1) == INVALID
        assert f(x=None) == f(c=None) == f(s=None) == INVALID
        assert f(x=ODD1) == f(x=ODD2, dt=0) == f(c=ODD8) == f(s=ODD8) == UNSUPPORTED
    assert rows(count=ODD2) == gated(count=ODD1) == dispatch(slot=ODD2) == columns(off=ODD2) == UNSUPPORTED
    assert dispatch(T=-1) == dispatch(K=0) == dispatch(T=1 << 30) == dispatch(slot=None) == INVALID
    assert columns(E=0) == columns(off=None) == INVALID and columns(E=257) == UNSUPPORTED
    assert rows(R=0, x=None) == gated(R=0, x=None) == dispatch(T=0, x=None) == columns(R=0, x=None) == OK


def test_weights_refuse(lib):
    def call(w=FAKE, E=2, N=64, H=64, dt=1, c=FAKE, s=FAKE, ct=FAKE, st=FAKE):
        return lib.eqb_quantize_weights(w, E, N, H, dt, c, s, ct, st, None)

    assert call(E=0) == call(N=0) == call(H=0) == call(N=(1 << 24) + 1) == call(dt=4) == call(w=None) == INVALID
    assert call(c=None) == call(s=None) == call(ct=None) == call(st=None) == call(c=None, s=None, ct=None, st=None) == INVALID
    assert call(E=257) == call(w=ODD1) == call(w=ODD2, dt=0) == call(c=ODD8) == call(s=ODD8) == call(ct=ODD8) == call(st=ODD8) == UNSUPPORTED
    assert call(E=256, N=1 << 24, H=1 << 24) == UNSUPPORTED          # more tiles than a launch has


def test_products_refuse(lib):
    def product(x=FAKE, xs=FAKE, w=FAKE, ws=FAKE, off=FAKE, R=64, E=3, N=64, H=64, dt=1, out=FAKE):
        return lib.eqb_experts_product(x, xs, w, ws, off, R, E, N, H, dt, out, None)

    def grad(x=FAKE, xs=FAKE, w=FAKE, ws=FAKE, off=FAKE, R=64, E=3, N=64, H=64, dt=1, out=FAKE):
        return lib.eqb_experts_grad_weight(x, xs, w, ws, off, R, E, N, H, dt, out, None)

    for f in (product, grad):
        assert f(R=-1) == f(R=1 << 31) == f(E=0) == f(N=0) == f(H=0) == f(H=(1 << 24) + 1) == f(N=(1 << 24) + 1) == f(dt=3) == INVALID
        assert f(E=257) == UNSUPPORTED
        assert f(x=None) == f(xs=None) == f(w=None) == f(ws=None) == f(off=None) == f(out=None) == INVALID
        assert f(x=ODD8) == f(xs=ODD8) == f(w=ODD8) == f(ws=ODD8) == f(off=ODD2) == f(out=ODD1) == f(out=ODD2, dt=0) == UNSUPPORTED
    assert product(R=0, x=None) == OK and grad(R=0, x=None) == INVALID        # zeros are written
    assert grad(R=1 << 24) == UNSUPPORTED


def test_gate_refuses(lib):
    def gate(x=FAKE, count=None, R=8, H=64, dt=1, h=FAKE):
        return lib.eqb_gated(x, count, R, H, dt, h, None)

    def back(g=FAKE, x=FAKE, count=None, R=8, H=64, dt=1, gx=FAKE):
        return lib.eqb_gated_backward(g, x, count, R, H, dt, gx, None)

    for f in (gate, back):
        assert f(R=-1) == f(R=1 << 31) == f(H=0) == f(H=(1 << 24) + 1) == f(dt=3) == f(x=None) == INVALID
        assert f(x=ODD1) == f(x=ODD2, dt=0) == f(count=ODD2) == UNSUPPORTED
        assert f(R=0, x=None) == OK
    assert gate(h=None) == back(g=None) == back(gx=None) == INVALID
    assert gate(h=ODD1) == back(g=ODD1) == back(gx=ODD2, dt=0) == UNSUPPORTED


def test_binding_refuses_before_the_call():
    from paper_2609_28053_amd import GatedExperts, ScoredRouter, eqb
    x = torch.zeros((4, 200))
    codes, scales = torch.zeros((4, 256), dtype=torch.uint8).view(eqb._CODES), torch.zeros((4, 4), dtype=torch.uint8).view(eqb._SCALES)
    with pytest.raises(ValueError, match="GPU"):
        eqb.eqb_quantize_rows(x, codes, scales)
    with pytest.raises(ValueError, match="GPU"):
        eqb._coded(codes, scales, (4,), 200, "")
    with pytest.raises(ValueError, match="shape"):           # codes of whole blocks
        eqb._coded(codes[:, :200], scales, (4,), 200, "")
    with pytest.raises(ValueError, match="shape"):
        eqb._coded(codes, scales[:, :2], (4,), 200, "")
    with pytest.raises(ValueError, match="shape"):
        eqb._coded(None, scales, (5,), 200, "")
    with pytest.raises(TypeError):
        eqb._logit_type(x.double())
    assert [eqb._logit_type(torch.zeros(1, dtype=t)) for t in (torch.float32, torch.bfloat16, torch.float16, torch.int16)] == [0, 1, 2, 1]
    with pytest.raises(ValueError, match="even"):
        eqb.eqb_gated_quantize(torch.zeros((4, 5)), codes, scales)
    off = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="codes has shape"):          # three rows of codes for four of out
        eqb.eqb_experts_product(codes[:3], scales, codes.view(1, 4, 256), scales, off, torch.zeros((4, 4)))
    with pytest.raises(ValueError, match="gradient's codes has shape"):
        eqb.eqb_experts_grad_weight(codes, scales, codes, scales, off, torch.zeros((1, 3, 4)))
    with pytest.raises(ValueError, match="not \\[E,2F,H\\]"):
        GatedExperts(torch.zeros((2, 6, 4)), torch.zeros((2, 4, 2)))
    with pytest.raises(ValueError, match="experts"):
        ScoredRouter(8, 2).forward(torch.zeros((4, 16)))
    with pytest.raises(KeyError):
        ScoredRouter(8, 2, score="tanh")
