"""eqb_gated_quantize_columns refuses wrong arguments before the HIP runtime is touched (no GPU)."""
import ctypes

import pytest
import torch

from test_experts_abi import FAKE, INVALID, LIB, ODD1, ODD2, ODD8, OK, UNSUPPORTED, V, i32, i64


def test_gated_columns_refuse():
    lib = ctypes.CDLL(LIB)
    lib.eqb_gated_quantize_columns.argtypes = [V, V, i64, i32, i32, i32, V, V, V]

    def call(x=FAKE, off=FAKE, R=8, E=3, H=64, dt=1, c=FAKE, s=FAKE):
        return lib.eqb_gated_quantize_columns(x, off, R, E, H, dt, c, s, None)

    assert call(R=-1) == call(R=1 << 31) == call(H=0) == call(H=(1 << 24) + 1) == call(dt=3) == call(dt=-1) == call(E=0) == INVALID
    assert call(x=None) == call(off=None) == call(c=None) == call(s=None) == INVALID
    assert call(E=257) == call(x=ODD1) == call(x=ODD2, dt=0) == call(off=ODD2) == call(c=ODD8) == call(s=ODD8) == UNSUPPORTED
    assert call(R=0, x=None) == OK


def test_binding_refuses():
    from paper_2609_28053_amd import eqb
    off = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="even"):
        eqb.eqb_gated_quantize_columns(torch.zeros((4, 5)), off, None, None)
    with pytest.raises(ValueError, match="GPU"):
        eqb.eqb_gated_quantize_columns(torch.zeros((4, 6)), off, None, None)
