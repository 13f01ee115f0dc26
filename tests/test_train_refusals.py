"""Arguments that the training operators' C ABI refuses without touching the GPU (CPU)."""
import ctypes

import pytest

from test_train_abi import FAKE, INVALID, ODD2, UNSUPPORTED, LIB, Tensor, V, f64, i32

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
