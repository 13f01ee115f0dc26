"""Biases whose group sums binary32 does not hold (its lowest and largest numbers, infinities), with rows that masks leave
little of: the choice of the binary64 oracle."""
import numpy as np
import pytest
import torch

from oracle import experts_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu
LOWEST = float(torch.finfo(torch.float32).min)


@pytest.mark.parametrize("softmax", [False, True])
@pytest.mark.parametrize("E,K,groups,keep", [(8, 2, 4, 3), (16, 8, 2, 1), (32, 1, 4, 3), (64, 13, 4, 1), (64, 6, 8, 4), (128, 6, 8, 3),
                                             (128, 16, 4, 2), (256, 8, 8, 4), (64, 20, 4, 2), (256, 5, 32, 9)])
def test_groups_of_large_biases(eqb, E, K, groups, keep, softmax):  # noqa: F811
    say(f"groups of large biases E={E} K={K} groups={groups},{keep} softmax={softmax}")
    rng = np.random.default_rng(E + K)
    T = 60
    for kind in ("lowest", "large", "all"):
        for masked in (0.0, 0.5, 0.95):
            z = rng.normal(size=(T, E)).astype(np.float32)
            z[rng.random((T, E)) < masked] = -np.inf
            b = {"lowest": np.where(rng.random(E) < 0.5, LOWEST, 0.0), "large": rng.choice([LOWEST, -2e38, 2e38, 3e38, -LOWEST, 0.0], size=E),
                 "all": rng.choice([-np.inf, np.inf, LOWEST, -LOWEST, 3e38, -3e38, 0.0, 1.0], size=E)}[kind]
            zt = torch.from_numpy(z).to(torch.bfloat16)
            bt = torch.from_numpy(b.astype(np.float32))
            idx, w = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
            eqb.eqb_route_scored(zt.cuda(), bt.cuda(), K, idx, w, eqb.EQB_SCORE_SOFTMAX if softmax else eqb.EQB_SCORE_SIGMOID,
                                 groups, keep, 2, True)
            want, _ = O.route(zt.to(torch.float64).numpy(), bt.numpy().astype(np.float64), K, softmax, groups, keep, 2)
            assert np.array_equal(idx.cpu().numpy(), want), (kind, masked)
