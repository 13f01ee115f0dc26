"""Streamed rows (calls on 256 MiB of experts' rows and more) that are whole lines of 128 bytes
but no whole segments: the last pieces of a row overlap ones before them, or lie past it.

Tolerance: dispatched rows are exact, a gradient row is one product rounded once, a combined
value two products and a sum in binary32 and one rounding, a weight's gradient sums H
products in any order (H 2^-24 of their magnitudes)."""
import pytest
import torch

from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)
from test_gpu_experts import plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H,dtype", [(70001, 1088, torch.bfloat16), (70001, 544, torch.float32), (9001, 8256, torch.float16),
                                       (30011, 2112, torch.bfloat16), (70001, 1984, torch.bfloat16)])
def test_partial_segments(eqb, T, H, dtype):  # noqa: F811
    K, E = 2, 8
    size = torch.empty((), dtype=dtype).element_size()
    K = K if T * K * H * size >= 256 << 20 else 3
    assert T * K * H * size >= 256 << 20 and H * size % 128 == 0 and H * size % 4096 != 0
    g = torch.Generator(device="cuda")
    g.manual_seed(H)
    idx = torch.rand((T, E), generator=g, device="cuda").topk(K, dim=1).indices.to(torch.int32)
    idx[::17, 0] = -1
    _, slot = plan(eqb, idx.cpu().numpy(), E)
    kept = slot >= 0
    at = torch.where(kept, slot, 0).long()
    say(f"streamed rows {T} x {H} {dtype}")
    x = torch.randn((T, H), generator=g, device="cuda", dtype=dtype)
    rows = torch.full((T * K, H), 7.0, dtype=dtype, device="cuda")
    eqb.eqb_dispatch(x, slot, rows)
    for k in range(K):
        assert torch.equal(rows[at[:, k]][kept[:, k]], x[kept[:, k]])
    assert bool((rows[int(kept.sum()):] == 7.0).all())           # rows that no slot names
    out = torch.randn((T * K, H), generator=g, device="cuda", dtype=dtype)
    w = torch.rand((T, K), generator=g, device="cuda")
    y = torch.empty_like(x)
    eqb.eqb_combine(out, slot, w, y)
    want, size = torch.zeros((T, H), dtype=torch.float64, device="cuda"), torch.zeros((T, H), dtype=torch.float64, device="cuda")
    for k in range(K):
        part = torch.where(kept[:, k:k + 1], w[:, k:k + 1].double() * out[at[:, k]].double(), 0.0)
        want += part
        size += part.abs()
    half = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 0.0}[dtype]
    assert bool(((y.double() - want).abs() <= (K + 1) * 2.0 ** -24 * size * (1 + half) + half * want.abs() + 2.0 ** -25).all())
    del want, size, part
    gr, gw = torch.full_like(out, 7.0), torch.empty_like(w)
    eqb.eqb_combine_backward(x, out, slot, w, gr, gw)
    for k in range(K):
        on = kept[:, k]
        assert torch.equal(gr[at[:, k]][on], (w[:, k:k + 1] * x.float()).to(dtype)[on])
        dot = x.double() * out[at[:, k]].double()
        far = (gw[:, k].double() - torch.where(on, dot.sum(1), 0.0)).abs()
        assert bool((far <= H * 2.0 ** -24 * dot.abs().sum(1)).all()) and bool((gw[:, k][~on] == 0).all())
    assert bool((gr[int(kept.sum()):] == 7.0).all())
