"""CPU oracle for the operators that train a layer around its routing.

TEST INFRASTRUCTURE ONLY, like ``eqb_oracle``: it shares no code, constant table
or helper with the HIP path.  Everything is computed in binary64 by numpy, from
the definitions:

* the balance loss of a group of n valid tokens, alpha sum_e F_e prob_e with
  F_e = E f_e / (K n) and prob_e the mean probability of expert e (arXiv
  2609.28053, Sec. 2, "GShard"), over normalised sigmoids or a softmax, and its
  gradient with the loads held fixed (App. D), plus the router backward with the
  injected term (Sec. 4);
* the experts' rows (Eq. 1): the stable order by expert, the gather, the weighted
  sum, and the gradients of both;
* one AdamW step, with binary64 states or with 8-bit ones: codes of E4M3 values
  (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7F no number) in blocks of
  256 with a scale each, rounded at random by given 16-bit numbers.
"""
import numpy as np

BLOCK = 256


# ------------------------------------------------------------ balance loss --
def probabilities(x, softmax):
    """p [T,E] of the logits x [T,E] (binary64; -inf allowed); rows of nothing but -inf: 0.  Normalised sigmoids are
    taken as exp(log sigmoid(x) - its maximum), so that no row underflows."""
    with np.errstate(invalid="ignore", over="ignore"):
        a = x if softmax else -np.logaddexp(0.0, -x)
    m = a.max(axis=1, keepdims=True)
    w = np.exp(a - np.where(np.isneginf(m), 0.0, m))
    d = w.sum(axis=1, keepdims=True)
    return np.divide(w, d, out=np.zeros_like(w), where=d > 0)


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def balance_loss(x, idx, K, alpha, part, valid=None, softmax=False, load=None):
    """loads [P,E], tokens [P], prob [P,E], loss [P]; idx may be None where load is given."""
    T, E = x.shape
    P = len(part) - 1
    ok = np.ones(T, dtype=bool) if valid is None else np.asarray(valid, dtype=bool)
    got = np.zeros((P, E), dtype=np.int64)
    tokens = np.zeros(P, dtype=np.int64)
    prob = np.zeros((P, E))
    loss = np.zeros(P)
    for p in range(P):
        rows = np.arange(part[p], part[p + 1])
        rows = rows[ok[rows]]
        tokens[p] = len(rows)
        if load is None:
            picks = idx[rows].reshape(-1)
            picks = picks[(picks >= 0) & (picks < E)]
            got[p] = np.bincount(picks, minlength=E)
        else:
            got[p] = load[p]
        if len(rows):
            prob[p] = probabilities(x[rows], softmax).sum(axis=0) / len(rows)
            loss[p] = alpha * float(np.sum(E * got[p] / (K * len(rows)) * prob[p]))
    return got, tokens, prob, loss


def balance_backward(x, load, tokens, K, alpha, grad_loss, part, idx=None, grad_score=None, inj=None, valid=None,
                     softmax=False):
    """grad_z [T,E]."""
    T, E = x.shape
    out = np.zeros((T, E))
    ok = np.ones(T, dtype=bool) if valid is None else np.asarray(valid, dtype=bool)
    for p in range(len(part) - 1):
        for t in range(part[p], part[p + 1]):
            if not ok[t]:
                continue
            row = x[t:t + 1]
            pr = probabilities(row, softmax)[0]
            F = E * load[p] / (K * tokens[p])
            g = alpha * grad_loss[p] / tokens[p] * pr * (F - float(pr @ F))
            if not softmax:
                g = g * sigmoid(-row[0])
            up = np.zeros(E) if inj is None else np.array(inj[p], dtype=np.float64)
            if idx is not None:
                for k in range(idx.shape[1]):
                    if 0 <= idx[t, k] < E:
                        up[idx[t, k]] += grad_score[t, k]
            out[t] = g + up * sigmoid(row[0]) * sigmoid(-row[0])
    return out


# ----------------------------------------------------------- experts' rows --
def dispatch_plan(idx, E):
    """offsets [E+1] and slot [T,K] by walking the pairs expert by expert."""
    T, K = idx.shape
    slot = np.full((T, K), -1, dtype=np.int64)
    offsets = [0]
    for e in range(E):
        for t, k in zip(*np.nonzero(idx == e)):          # row-major: ascending t*K + k
            slot[t, k] = offsets[-1] + np.count_nonzero(slot[idx == e] >= 0)
        offsets.append(offsets[-1] + int(np.count_nonzero(idx == e)))
    return np.array(offsets), slot


def dispatch(x, slot, rows):
    out = np.array(rows, dtype=np.float64)
    for t, k in np.ndindex(*slot.shape):
        if 0 <= slot[t, k] < len(out):
            out[slot[t, k]] = x[t]
    return out


def combine(rows, slot, weight, H):
    T, K = slot.shape
    y = np.zeros((T, H))
    for t, k in np.ndindex(T, K):
        if 0 <= slot[t, k] < len(rows):
            y[t] += (1.0 if weight is None else float(weight[t, k])) * rows[slot[t, k]]
    return y


def combine_backward(grad_y, rows, slot, weight, grad_rows):
    g = np.array(grad_rows, dtype=np.float64)
    gw = np.zeros(slot.shape)
    for t, k in np.ndindex(*slot.shape):
        r = slot[t, k]
        if 0 <= r < len(rows):
            g[r] = float(weight[t, k]) * grad_y[t]
            gw[t, k] = float(np.dot(grad_y[t], rows[r]))
    return g, gw


# ------------------------------------------------------------------- AdamW --
def e4m3_values():
    """The values of the 256 codes; NaN for the two patterns that stand for none."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = np.nan if (c & 0x7F) == 0x7F else (-v if c & 0x80 else v)
    return out


E4M3 = e4m3_values()


def round_e4m3(y, rnd16):
    """Codes of 0 <= y <= 448: the code at or below y, or the next one where y's place between them plus rnd16/65536
    reaches 1."""
    grid = E4M3[:127]                                   # ascending, codes 0..126
    low = np.clip(np.searchsorted(grid, y, side="right") - 1, 0, 126)
    high = np.minimum(low + 1, 126)
    gap = grid[high] - grid[low]
    frac = np.divide(y - grid[low], gap, out=np.zeros_like(y), where=gap > 0)
    return np.where(frac + rnd16 / 65536.0 >= 1.0, high, low)


def quantise(x, rnd16, nonzero):
    """Codes and scales (binary64) of a tensor in blocks of 256 by its magnitude, the sign put on top; nonzero: a value
    above 0 does not become 0."""
    n = len(x)
    codes = np.zeros(n, dtype=np.int64)
    scales = []
    for b in range(0, n, BLOCK):
        a = np.abs(x[b:b + BLOCK])
        top = a.max()
        s = 0.0 if top < 2.0 ** -100 else top / 448.0
        scales.append(s)
        if s == 0.0:
            continue
        c = round_e4m3(np.minimum(a / s, 448.0), rnd16[b:b + BLOCK])
        codes[b:b + BLOCK] = np.where(nonzero & (a > 0) & (c == 0), 1, c)
    return codes + 128 * np.signbit(x), np.array(scales)


def dequantise(codes, scales):
    return E4M3[codes] * np.repeat(scales, BLOCK)[:len(codes)]


def tensor_key(seed, step, i):
    """The 32 bits that a tensor's random numbers of a step start from."""
    M = (1 << 64) - 1
    k = (seed + step * 0x9E3779B97F4A7C15 + i * 0xD1B54A32D192ED03) & M
    k = ((k ^ (k >> 32)) * 0xBF58476D1CE4E5B9) & M
    k = ((k ^ (k >> 29)) * 0x94D049BB133111EB) & M
    return (k ^ (k >> 32)) & 0xFFFFFFFF


def random32(n, key, start=0):
    """32 random bits of elements start .. start + n - 1 of a tensor with that key."""
    mul = lambda v, c: (v * np.uint64(c)) & np.uint64(0xFFFFFFFF)  # noqa: E731
    j = np.arange(n, dtype=np.uint64) + np.uint64(start)
    x = ((j + np.uint64(key)) & np.uint64(0xFFFFFFFF)) ^ mul(j >> np.uint64(32), 0x9E3779B1)
    x = mul(x ^ (x >> np.uint64(16)), 0x7FEB352D)
    x = mul(x ^ (x >> np.uint64(15)), 0x846CA68B)
    return (x ^ (x >> np.uint64(16))).astype(np.int64)


def adamw(w, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """New w, m, v of one step in binary64."""
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    update = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return w * (1 - lr * weight_decay) - lr * update, m, v


def adamw32(w, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """The same in the binary32 operations that the interface states, one by one: new w, m, v and sqrt(v)."""
    f = np.float32
    w, g, m, v = (np.asarray(a, dtype=f) for a in (w, g, m, v))
    g = g * f(grad_scale)
    m = m * f(beta1) + g * f(1 - beta1)
    v = v * f(beta2) + (g * f(1 - beta2)) * g
    r = np.sqrt(v)
    d = r * f(1 / np.sqrt(1 - beta2 ** step)) + f(eps)
    w = w * f(1 - lr * weight_decay) - (m / d) * f(lr / (1 - beta1 ** step))
    return w, m, v, r
