"""Arguments that the training operators' C ABI refuses without touching the GPU (CPU)."""
import ctypes

import pytest

from test_train_abi import FAKE, INVALID, LIB, ODD1, ODD2, UNSUPPORTED, Tensor, V, f64, i32, lib as abi  # noqa: F401

@pytest.fixture(scope="module")
def lib():
    lib = ctypes.CDLL(LIB)
    lib.eqb_adamw_step_counted.argtypes = [V, i32, i32, i32, V, f64, f64, f64, f64, ctypes.c_uint64, V, V, V]
    return lib


def test_a_counted_step_refuses(lib):
    a = 0x10000

    def call(counter=FAKE, n=1, dt=0, bits=32, lr=1e-3, b2=0.99, **kw):
        t = dict(param=a, grad=a, copy=None, m=a, v=a, ms=None, vs=None, numel=10, wd=0.1)
        t.update(kw)
        arr = (Tensor * 1)(Tensor(**t))
        return lib.eqb_adamw_step_counted(ctypes.cast(arr, V), n, dt, bits, counter, lr, 0.9, b2, 1e-8, 0, None, None, None)

    assert call(counter=None) == call(n=-1) == call(dt=2) == call(bits=16) == INVALID
    assert call(lr=float("nan")) == call(b2=1.0) == call(param=None) == call(bits=8) == INVALID
    assert call(counter=ODD2) == call(counter=V(0x10004)) == call(m=a + 1) == UNSUPPORTED


def test_32_bit_arguments_off_their_alignment_are_refused(abi):  # noqa: F811
    """Scalar loads drop an address's last two bits, so such an argument would read or write its neighbours."""
    need, plan = abi.eqb_balance_workspace_size(8, 1), abi.eqb_dispatch_workspace_size(100000, 2, 8)

    def loss(idx=FAKE, load=FAKE, tokens=FAKE, prob=FAKE, loss=FAKE):
        return abi.eqb_balance_loss(FAKE, idx, None, 64, 8, 2, None, 1, 0, 0.1, load, tokens, prob, loss, FAKE, need, None)

    def grad(load=FAKE, tokens=FAKE, gl=FAKE, idx=FAKE, gs=FAKE, inj=FAKE):
        return abi.eqb_balance_backward(FAKE, load, tokens, gl, idx, gs, inj, None, 64, 8, 2, None, 1, 0, 0.1, FAKE, None)

    def order(idx=FAKE, off=FAKE, slot=FAKE):
        return abi.eqb_dispatch_plan(idx, 100000, 2, 8, off, slot, FAKE, plan, None)

    def adamw(scale=None, inf=None):
        a = 0x10000
        arr = (Tensor * 1)(Tensor(param=a, grad=a, copy=None, m=a, v=a, ms=None, vs=None, numel=10, wd=0.1))
        return abi.eqb_adamw_step(ctypes.cast(arr, V), 1, 0, 32, 1, 1e-3, 0.9, 0.99, 1e-8, 0, scale, inf, None)

    for odd in (ODD1, ODD2):
        assert loss(idx=odd) == loss(load=odd) == loss(tokens=odd) == loss(prob=odd) == loss(loss=odd) == UNSUPPORTED
        assert grad(load=odd) == grad(tokens=odd) == grad(gl=odd) == grad(idx=odd) == grad(gs=odd) == grad(inj=odd) == UNSUPPORTED
        assert order(idx=odd) == order(off=odd) == order(slot=odd) == UNSUPPORTED
        assert abi.eqb_dispatch(FAKE, odd, 4, 2, 8, 16, 1, FAKE, None) == UNSUPPORTED
        assert abi.eqb_combine(FAKE, odd, None, 4, 2, 8, 16, 1, FAKE, None) == UNSUPPORTED
        assert abi.eqb_combine(FAKE, FAKE, odd, 4, 2, 8, 16, 1, FAKE, None) == UNSUPPORTED
        for k in range(3):
            p = [odd if i == k else FAKE for i in range(3)]
            assert abi.eqb_combine_backward(FAKE, FAKE, p[0], p[1], 4, 2, 8, 16, 1, FAKE, p[2], None) == UNSUPPORTED
        assert adamw(scale=odd) == adamw(inf=odd) == UNSUPPORTED
