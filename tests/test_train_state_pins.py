"""The recipe that tells rounding at random from rounding to nearest, on the oracle (CPU): the
states of the first follow the exact ones, those of the second do not, and weights that do
not move are seen."""
import numpy as np

import state_recipe as S
from oracle import train_oracle as O


def run(random):
    m, r, g, counts = S.start()
    half = np.full(S.N, 32768)
    cm, sm = O.quantise(m, half, False)
    cr, sr = O.quantise(r, half, True)
    assert np.all(O.E4M3[cm][counts] == 160) and np.all(O.E4M3[cr][counts] == 112)      # exact codes
    w = np.zeros(S.N)
    for step in range(S.FIRST, S.FIRST + S.STEPS):
        m, r = O.dequantise(cm, sm), O.dequantise(cr, sr)
        w, m, _, r = O.adamw32(w, g, m, r * r, step, S.LR, S.BETA1, S.BETA2, S.EPS, 0.0)
        rnd = O.random32(S.N, O.tensor_key(5, step, 0)) if random else None
        cm, sm = O.quantise(m.astype(np.float64), rnd & 0xFFFF if random else half, False)
        cr, sr = O.quantise(r.astype(np.float64), rnd >> 16 if random else half, True)
    return O.dequantise(cm, sm)[counts], (O.dequantise(cr, sr) ** 2)[counts], w.astype(np.float64)[counts]


def test_rounding_at_random_follows():
    m, v, w = run(True)
    assert S.m_follows(m) and S.v_follows(v) and S.w_follows(w)


def test_rounding_to_nearest_and_resting_weights_are_seen():
    m, v, w = run(False)
    assert not S.m_follows(m) and not S.v_follows(v)
    assert np.allclose(m, S.M0, rtol=1e-5) and np.allclose(v, S.R0 ** 2, rtol=1e-5)     # frozen
    assert not S.w_follows(np.zeros_like(w))
