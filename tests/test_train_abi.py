"""The training operators' C ABI without a GPU: every wrong argument is refused before
the HIP runtime is touched, and the binding refuses what it can see."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.environ.get("EQB_LIB", os.path.join(ROOT, "paper_2609_28053_amd", "libeqb.so"))
OK, INVALID, UNSUPPORTED = 0, 1, 2
V, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double
FAKE = V(0x10000)       # never dereferenced: the calls below fail their checks first
ODD2 = V(0x10002)
ODD1 = V(0x10001)


@pytest.fixture(scope="module")
def lib():
    lib = ctypes.CDLL(LIB)
    lib.eqb_balance_workspace_size.argtypes = [i32, i32]
    lib.eqb_balance_workspace_size.restype = ctypes.c_size_t
    lib.eqb_balance_loss.argtypes = [V, V, V, i64, i32, i32, V, i32, i32, f64, V, V, V, V, V, ctypes.c_size_t, V]
    lib.eqb_balance_backward.argtypes = [V] * 8 + [i64, i32, i32, V, i32, i32, f64, V, V]
    lib.eqb_dispatch_workspace_size.argtypes = [i64, i32, i32]
    lib.eqb_dispatch_workspace_size.restype = ctypes.c_size_t
    lib.eqb_dispatch_plan.argtypes = [V, i64, i32, i32, V, V, V, ctypes.c_size_t, V]
    lib.eqb_dispatch.argtypes = [V, V, i64, i32, i64, i32, i32, V, V]
    lib.eqb_combine.argtypes = [V, V, V, i64, i32, i64, i32, i32, V, V]
    lib.eqb_combine_backward.argtypes = [V, V, V, V, i64, i32, i64, i32, i32, V, V, V]
    lib.eqb_adamw_step.argtypes = [V, i32, i32, i32, i64, f64, f64, f64, f64, ctypes.c_uint64, V, V, V]
    return lib


def table(*off):
    arr = (i64 * len(off))(*off)
    return ctypes.cast(arr, V), arr


def test_balance_loss_refuses(lib):
    need = lib.eqb_balance_workspace_size(8, 1)
    assert need > 0 and lib.eqb_balance_workspace_size(12, 1) == 0 and lib.eqb_balance_workspace_size(8, 257) == 0
    assert lib.eqb_balance_workspace_size(8, 0) == 0

    def call(z=FAKE, T=64, E=8, K=2, po=None, P=1, score=0, alpha=0.1, load=FAKE, tokens=FAKE, prob=FAKE, loss=FAKE,
             ws=FAKE, size=need):
        return lib.eqb_balance_loss(z, FAKE, None, T, E, K, po, P, score, alpha, load, tokens, prob, loss, ws, size, None)

    assert call(T=-1) == call(T=1 << 31) == call(K=0) == call(K=8) == INVALID
    assert call(E=12) == call(E=512) == UNSUPPORTED
    assert call(score=2) == call(score=-1) == call(alpha=float("nan")) == INVALID
    assert call(z=None) == call(load=None) == call(tokens=None) == call(prob=None) == call(loss=None) == INVALID
    assert call(ws=None) == call(size=need - 1) == INVALID
    assert call(z=V(0x10008)) == call(ws=V(0x10010)) == UNSUPPORTED
    assert call(P=2) == INVALID
    po, keep = table(0, 40, 30, 64)
    assert call(po=po, P=3) == INVALID


def test_balance_backward_refuses(lib):
    def call(z=FAKE, load=FAKE, tokens=FAKE, gl=FAKE, idx=None, gs=None, T=64, E=8, K=2, P=1, score=0, alpha=0.1, gz=FAKE):
        return lib.eqb_balance_backward(z, load, tokens, gl, idx, gs, None, None, T, E, K, None, P, score, alpha, gz, None)

    assert call(T=-1) == call(K=0) == call(K=8) == call(score=3) == call(alpha=float("nan")) == call(P=2) == INVALID
    assert call(E=7) == UNSUPPORTED
    assert call(z=None) == call(load=None) == call(tokens=None) == call(gl=None) == call(gz=None) == INVALID
    assert call(idx=FAKE) == call(gs=FAKE) == INVALID            # one without the other
    assert call(z=V(0x10008)) == call(gz=V(0x10008)) == UNSUPPORTED
    assert call(T=0) == OK


def test_dispatch_plan_refuses(lib):
    size = lib.eqb_dispatch_workspace_size
    assert size(1, 2, 8) == 0 and size(-1, 2, 8) == 0 and size(1 << 30, 2, 8) == 0 and size(100000, 2, 12) == 0
    need = size(100000, 2, 8)
    assert need > 0

    def call(idx=FAKE, T=100000, K=2, E=8, off=FAKE, slot=FAKE, ws=FAKE, n=need):
        return lib.eqb_dispatch_plan(idx, T, K, E, off, slot, ws, n, None)

    assert call(T=-1) == call(K=0) == call(K=8) == call(T=1 << 30) == INVALID
    assert call(E=24) == UNSUPPORTED
    assert call(idx=None) == call(off=None) == call(slot=None) == call(ws=None) == call(n=need - 1) == INVALID
    assert call(ws=V(0x10008)) == UNSUPPORTED


def test_rows_refuse(lib):
    def dispatch(x=FAKE, slot=FAKE, T=4, K=2, R=8, H=16, dt=1, out=FAKE):
        return lib.eqb_dispatch(x, slot, T, K, R, H, dt, out, None)

    def combine(rows=FAKE, slot=FAKE, T=4, K=2, R=8, H=16, dt=1, y=FAKE):
        return lib.eqb_combine(rows, slot, None, T, K, R, H, dt, y, None)

    def back(gy=FAKE, rows=FAKE, slot=FAKE, w=FAKE, T=4, K=2, R=8, H=16, dt=1, gr=FAKE, gw=FAKE):
        return lib.eqb_combine_backward(gy, rows, slot, w, T, K, R, H, dt, gr, gw, None)

    for f in (dispatch, combine, back):
        assert f(T=-1) == f(K=0) == f(R=-1) == f(R=1 << 31) == f(H=0) == f(dt=3) == f(dt=-1) == INVALID
        assert f(T=1 << 30) == f(slot=None) == INVALID
        assert f(T=0, slot=None) == OK
    assert dispatch(x=None) == dispatch(out=None) == combine(rows=None) == combine(y=None) == INVALID
    assert back(gy=None) == back(rows=None) == back(w=None) == back(gr=None) == back(gw=None) == INVALID
    assert dispatch(x=ODD1) == dispatch(x=ODD2, dt=0) == combine(y=ODD1) == back(gr=ODD2, dt=0) == UNSUPPORTED


class Tensor(ctypes.Structure):
    _fields_ = [(n, V) for n in ("param", "grad", "copy", "m", "v", "ms", "vs")] + [("numel", i64), ("wd", f64)]


def test_adamw_refuses(lib):
    a = 0x10000

    def call(n=1, dt=0, bits=32, step=1, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, null=False, more=None, **kw):
        t = dict(param=a, grad=a, copy=None, m=a, v=a, ms=None, vs=None, numel=10, wd=0.1)
        t.update(kw)
        tensors = [t] + ([dict(t, **more)] if more else [])
        arr = (Tensor * len(tensors))(*[Tensor(**x) for x in tensors])
        return lib.eqb_adamw_step(None if null else ctypes.cast(arr, V), len(tensors) if more else n, dt, bits, step, lr,
                                  b1, b2, eps, 0, None, None, None)

    nan = float("nan")
    assert call(n=-1) == call(null=True) == call(dt=2) == call(bits=16) == call(step=0) == INVALID
    assert call(lr=nan) == call(b1=1.0) == call(b1=-0.1) == call(b2=1.0) == call(b2=nan) == call(eps=-1.0) == INVALID
    assert call(param=None) == call(grad=None) == call(m=None) == call(v=None) == call(wd=nan) == INVALID
    assert call(numel=-1) == call(numel=(1 << 33) + 1) == INVALID
    assert call(bits=8) == call(bits=8, ms=a) == INVALID                     # scales missing
    assert call(more=dict(copy=a)) == call(copy=a, more=dict(copy=None)) == INVALID   # copies of some only
    assert call(param=a + 2) == call(m=a + 1) == call(grad=a + 2) == call(copy=a + 1) == UNSUPPORTED
    assert call(dt=1, grad=a + 1) == call(bits=8, ms=a + 2, vs=a) == UNSUPPORTED
    assert call(n=0) == call(n=0, null=True) == OK
    assert call(numel=0, param=None, grad=None, m=None, v=None) == OK


def test_binding_refuses_before_the_call():
    import torch

    from paper_2609_28053_amd import eqb
    cpu = torch.zeros(4)
    with pytest.raises(ValueError):          # no GPU tensor
        eqb.AdamwTensors([cpu], [cpu], [cpu], [cpu])
    with pytest.raises(ValueError):
        eqb.eqb_dispatch(cpu.view(2, 2), torch.zeros((2, 1), dtype=torch.int32), cpu.view(2, 2))
    with pytest.raises(TypeError):           # no type of gradients
        eqb._row_type(cpu.double(), "x")
    with pytest.raises(ValueError):
        eqb.AdamwTensors([], [], [], [], exp_avg_scale=[])
    eqb.eqb_adamw_step(eqb.AdamwTensors([], [], [], []), 1, 1e-3, stream=0)
