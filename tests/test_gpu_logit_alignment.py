"""Logits at every address that the header allows: 16 bytes past a multiple of 32, 64 and 128."""
import pytest
import torch

from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("E,K,groups", [(8, 3, 1), (32, 4, 4), (256, 8, 8), (64, 20, 1), (256, 7, 32)])
def test_logits_sixteen_bytes_along(eqb, dtype, E, K, groups):  # noqa: F811
    say(f"logits along E={E} K={K} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(E)
    T = 70
    z = torch.randn((T, E), generator=g, device="cuda").to(dtype)
    bias, gw = torch.randn(E, generator=g, device="cuda") * 0.1, torch.randn((T, K), generator=g, device="cuda")
    keep, pair = max(1, groups // 2), 2 if E // groups > 1 else 1

    def run(z, score, normalize):
        idx, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
        gz = torch.empty((T, E), device="cuda")
        eqb.eqb_route_scored(z, bias, K, idx, w, score, groups, keep, pair, normalize)
        eqb.eqb_route_scored_backward(z, idx, gw, gz, score, normalize)
        return idx, w, gz

    for score, normalize in ((eqb.EQB_SCORE_SIGMOID, True), (eqb.EQB_SCORE_SOFTMAX, True), (eqb.EQB_SCORE_SOFTMAX, False)):
        want = run(z, score, normalize)
        for past in (16, 48, 112):
            n = past // z.element_size()
            flat = torch.empty(z.numel() + n, dtype=dtype, device="cuda")
            along = flat[n:].view(T, E)
            along.copy_(z)
            assert along.data_ptr() % 32 == 16
            assert all(torch.equal(a, b) for a, b in zip(want, run(along, score, normalize)))
