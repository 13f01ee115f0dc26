"""8-bit states on the GPU: moments that move by a small part of a code a step follow the exact
ones (rounding to nearest would leave them where they are; the recipe's bounds, and that they
see this, are pinned on the CPU)."""
import numpy as np
import pytest
import torch

import state_recipe as S
from oracle import train_oracle as O
from test_gpu_balance import eqb, say  # noqa: F401 (eqb is a fixture)

pytestmark = pytest.mark.gpu


def test_slow_moments_follow_the_exact_ones(eqb):  # noqa: F811
    m, r, g, counts = S.start()
    half = np.full(S.N, 32768)
    state = []
    for x, nonzero in ((m, False), (r, True)):
        codes, scales = O.quantise(x, half, nonzero)
        state.append(torch.from_numpy(codes.astype(np.uint8)).cuda().view(torch.float8_e4m3fn))
        state.append(torch.from_numpy(scales.astype(np.float32)).cuda())
    w, grad = torch.zeros(S.N, device="cuda"), torch.from_numpy(g.astype(np.float32)).cuda()
    table = eqb.AdamwTensors([w], [grad], [state[0]], [state[2]], exp_avg_scale=[state[1]], exp_avg_sq_scale=[state[3]])
    say("adamw, 500 steps of slow moments")
    for step in range(S.FIRST, S.FIRST + S.STEPS):
        eqb.eqb_adamw_step(table, step, S.LR, S.BETA1, S.BETA2, S.EPS, seed=5)
    end = [(c.to(torch.float32).double() * s.double().repeat_interleave(256)).cpu().numpy()[counts]
           for c, s in (state[:2], state[2:])]
    say(f"means: m {end[0].mean():.5f}, v {np.mean(end[1] ** 2):.5f}, w {float(w.mean()):.5f}")
    assert S.m_follows(end[0]) and S.v_follows(end[1] ** 2)
    assert S.w_follows(w.double().cpu().numpy()[counts])
