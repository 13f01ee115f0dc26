"""8-bit optimizer states that have to move by far less than half a code a step, and what
their means have to be at the end.

Every block of 256 starts with an element whose gradient is 1 and whose states are 1, the
block's largest, so that the scales stay 1/448; the other elements have m = 160/448,
sqrt(v) = 112/448 (both exact codes) and the gradient 1/2 from then on, for 500 steps of
beta1 = 0.9, beta2 = 0.999.  A step moves m by 6.4/448 at first, where codes are 16/448
apart, and sqrt(v) by 0.17/448, where they are 8/448 apart: rounding to nearest moves
neither, ever.

m: rounding that is right on average leaves its mean at 1/2 (less 0.15 0.9^500).  A step's
rounding has a variance of a quarter of the spacing's square at most, (8/448)^2, the mean
over time 1/(1 - 0.9^2) times that: 0.041 an element, 3.2e-4 the mean of 16,320.
v: exactly, b/16 + (1 - b)/4 with b = 0.999^500.  Rounding sqrt(v) = r up by a spacing D with
probability d/D (d: what the step moves r by) adds d D at most to the mean of v, where the
step itself moves it by 2 r d; D is r/8 at most: the growth is up to 1/16 larger.  r at the
end has a deviation of sqrt(sum d D) = sqrt((0.37 - 0.25) 0.37/8) = 0.074 at most, v one of
2 0.37 0.074 = 0.055, the mean 4.3e-4, which is 0.6% of the growth 0.0738.
w: minus the sum of m/r.  Its mean over the elements follows the exact one to the mean of 1/r
(r off by 3% and spread by 0.074/0.37 of itself, 4% of the mean of 1/r) and the correlation
of m and r, which share no rounding: 10%."""
import numpy as np

N, STEPS, FIRST = 64 * 256, 500, 10000
LR, BETA1, BETA2, EPS = 1e-3, 0.9, 0.999, 1e-8
M0, R0 = 160.0 / 448, 112.0 / 448


def start():
    """m, sqrt(v) and the gradient of every step (binary64), and which elements count."""
    counts = np.arange(N) % 256 != 0
    fill = lambda x: np.where(counts, x, 1.0)  # noqa: E731
    return fill(M0), fill(R0), fill(0.5), counts


def exact():
    """Means at the end without rounding: m, v and w."""
    m, v, w = M0, R0 * R0, 0.0
    for step in range(FIRST, FIRST + STEPS):
        m = BETA1 * m + (1 - BETA1) * 0.5
        v = BETA2 * v + (1 - BETA2) * 0.25
        w -= LR * (m / (1 - BETA1 ** step)) / (np.sqrt(v / (1 - BETA2 ** step)) + EPS)
    return m, v, w


def m_follows(m):
    return abs(float(np.mean(m)) - exact()[0]) <= 5 * 3.2e-4


def v_follows(v):
    growth = (float(np.mean(v)) - R0 * R0) / (exact()[1] - R0 * R0)
    return 1 - 5 * 0.006 <= growth <= 1 + 1 / 16 + 5 * 0.006


def w_follows(w):
    want = exact()[2]
    return abs(float(np.mean(w)) - want) <= 0.1 * abs(want)
