"""CPU oracle for the routing by scores and the experts' products in 8 bits.

TEST INFRASTRUCTURE ONLY, like ``eqb_oracle``: it shares no code, constant table
or helper with the HIP path.  Everything is computed in binary64 by numpy, from
the definitions:

* the choice of K experts by score plus bias within the best groups, one expert
  at a time, the weights, and their gradient with the choice held fixed;
* E4M3 codes (sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7F and 0xFF no
  number) of blocks of 128 with a power of two each, found from the table of all
  codes' values: of rows, of an expert's columns, of weights;
* the products of what codes and scales stand for, and the gated activation with
  its gradient.
"""
import numpy as np

BLOCK = 128


# ------------------------------------------------------------------ routing --
def scores(z, softmax):
    """Scores [T,E] of the logits z [T,E] (binary64; -inf: masked); rows of nothing but -inf: 0."""
    if not softmax:
        e = np.exp(-np.abs(z))
        return np.where(z >= 0, 1 / (1 + e), e / (1 + e))
    m = z.max(1, keepdims=True)
    e = np.exp(z - np.where(np.isneginf(m), 0.0, m))
    d = e.sum(1, keepdims=True)
    return np.divide(e, d, out=np.zeros_like(e), where=d > 0)


def shares(z, s, softmax):
    """What the chosen scores s of the logits z are of their sum: from their logarithms, so that scores that binary64
    does not hold have a share too (0 of masked ones and of none)."""
    on = z > -np.inf
    if not on.any():
        return np.zeros_like(s)
    x = z[on]
    log = x if softmax else x - np.logaddexp(0.0, x)
    r = np.exp(log - log.max())
    out = np.zeros_like(s)
    out[on] = r / r.sum()
    return out


def route(z, bias, K, softmax=False, groups=1, top_groups=1, group_top=1, normalize=True, scale=1.0):
    """idx [T,K] and weight [T,K]."""
    T, E = z.shape
    s = scores(z, softmax)
    idx, weight = np.full((T, K), -1), np.zeros((T, K))
    b = np.zeros(E) if bias is None else bias.astype(np.float64)
    each = E // groups
    for t in range(T):
        q = {e: s[t, e] + b[e] for e in range(E) if z[t, e] > -np.inf and s[t, e] + b[e] > -np.inf}
        if top_groups < groups:
            value = []
            for g in range(groups):
                mine = sorted((q[e] for e in range(g * each, (g + 1) * each) if e in q), reverse=True)
                value.append(sum(mine[:group_top]) if mine else -np.inf)
            kept = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
            q = {e: v for e, v in q.items() if e // each in kept}
        # without a bias the scores' order is the logits', also where the scores are no longer told apart
        best = sorted(q, key=lambda e: (-z[t, e] if bias is None else -q[e], e))[:K]
        idx[t, :len(best)] = best
        weight[t, :len(best)] = shares(z[t, best], s[t, best], softmax) if normalize else s[t, best]
    return idx, scale * weight


def route_backward(z, idx, g, softmax=False, normalize=True, scale=1.0):
    """grad_z [T,E] and a bound of the magnitudes that it is the sum of."""
    T, E = z.shape
    s = scores(z, softmax)
    grad, size = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        on = [k for k in range(idx.shape[1]) if 0 <= idx[t, k] < E]
        sk = s[t, idx[t, on]]
        gk = g[t, on]
        if normalize:
            r = shares(z[t, idx[t, on]], sk, softmax)
            x = z[t, idx[t, on]]
            rest = 1.0 if softmax else np.exp(-np.logaddexp(0.0, x))
            np.add.at(grad[t], idx[t, on], scale * (gk - gk @ r) * r * rest)
            np.add.at(size[t], idx[t, on], abs(scale) * (np.abs(gk) + np.abs(gk) @ r) * r * rest)
            continue
        a, m = scale * gk, abs(scale) * np.abs(gk)
        at, mt = np.zeros(E), np.zeros(E)
        np.add.at(at, idx[t, on], a)
        np.add.at(mt, idx[t, on], m)
        if softmax:
            grad[t] = s[t] * (at - a @ sk)
            size[t] = s[t] * (mt + m @ sk)
        else:
            with np.errstate(over="ignore"):
                rest = np.where(z[t] >= 0, np.exp(-np.abs(z[t])) / (1 + np.exp(-np.abs(z[t]))), 1 / (1 + np.exp(-np.abs(z[t]))))
            grad[t], size[t] = at * s[t] * rest, mt * s[t] * rest
    return grad, size


# ------------------------------------------------------------------ codes --
def code_values():
    """What the 256 codes stand for."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = (np.nan if (c & 127) == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)) * (-1 if c & 128 else 1)
    return v


VALUES = code_values()
_POSITIVE = VALUES[:127]


def encode(y):
    """The nearest codes of y (|y| <= 448, or no number), ties to the even code."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up = _POSITIVE[hi] - a
    down = a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(_POSITIVE[lo] == a, lo, code)
    return np.where(np.isfinite(y), np.where(np.signbit(y), code + 128, code), 127).astype(np.uint8)


def exponent(block):
    """The least x >= -126 with no finite value of the block above 448 2^x."""
    top = max((abs(v) for v in block.ravel() if np.isfinite(v)), default=0.0)
    x = -126
    while top > 448 * 2.0 ** x:
        x += 1
    return x


def quantize_rows(v):
    """codes [R,W], scales [R,S] (bytes) of v [R,H]."""
    R, H = v.shape
    blocks = -(-H // BLOCK)
    codes, scales = np.zeros((R, blocks * BLOCK), np.uint8), np.zeros((R, -(-blocks // 4) * 4), np.uint8)
    for j in range(blocks):
        part = v[:, j * BLOCK:(j + 1) * BLOCK]
        top = np.where(np.isfinite(part), np.abs(part), 0).max(1) if part.size else np.zeros(R)
        with np.errstate(divide="ignore"):
            x = np.maximum(np.ceil(np.log2(top / 448)), -126)
        for r in range(R):                      # the logarithm is only where to begin
            x[r] = -126 if top[r] == 0 else x[r]
            while x[r] > -126 and top[r] <= 448 * 2.0 ** (x[r] - 1):
                x[r] -= 1
            while top[r] > 448 * 2.0 ** x[r]:
                x[r] += 1
        codes[:, j * BLOCK:j * BLOCK + part.shape[1]] = encode(np.ldexp(part, -x[:, None].astype(int)))
        scales[:, j] = x + 127
    return codes, scales


def columns(rows, offsets):
    """First column of each expert and the width."""
    E = len(offsets) - 1
    return [BLOCK * (int(offsets[e]) // BLOCK + e) for e in range(E)], BLOCK * (rows // BLOCK + E)


def quantize_columns(v, offsets, codes, scales):
    """In place: codes [H,W] and scales of the experts' columns of v [R,H]."""
    starts, _ = columns(v.shape[0], offsets)
    for e, a in enumerate(starts):
        n = int(offsets[e + 1] - offsets[e])
        if n:
            c, s = quantize_rows(v[offsets[e]:offsets[e + 1]].T.copy())
            codes[:, a:a + c.shape[1]] = c
            scales[:, a // BLOCK:a // BLOCK + -(-n // BLOCK)] = s[:, :-(-n // BLOCK)]
    return codes, scales


def quantize_weights(w):
    """codes [E,N,W], scales [E,ceil(N/128),S] of w [E,N,H]."""
    E, N, H = w.shape
    nb, hb = -(-N // BLOCK), -(-H // BLOCK)
    codes, scales = np.zeros((E, N, hb * BLOCK), np.uint8), np.zeros((E, nb, -(-hb // 4) * 4), np.uint8)
    for e in range(E):
        for i in range(nb):
            for j in range(hb):
                part = w[e, i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
                x = exponent(part)
                codes[e, i * BLOCK:i * BLOCK + part.shape[0], j * BLOCK:j * BLOCK + part.shape[1]] = encode(np.ldexp(part, -x))
                scales[e, i, j] = x + 127
    return codes, scales


def decode(codes, scales):
    """What codes [...,W] with scales [...,S] stand for."""
    blocks = codes.shape[-1] // BLOCK
    power = np.exp2(scales[..., :blocks].astype(np.float64) - 127)
    return VALUES[codes] * np.repeat(power, BLOCK, axis=-1)


def decode_weights(codes, scales):
    return decode(codes, np.repeat(scales, BLOCK, axis=1)[:, :codes.shape[1]])


# ---------------------------------------------------------------- the gate --
def gated(x):
    """h [R,F] of x [R,2F] = (g, u)."""
    g, u = np.split(x, 2, axis=1)
    return g * scores(g, False) * u


def gated_backward(grad_h, x):
    """grad_x [R,2F] and the sizes of what it is the product of."""
    g, u = np.split(x, 2, axis=1)
    s, rest = scores(g, False), scores(-g, False)
    grad = np.concatenate([grad_h * u * s * (1 + g * rest), grad_h * g * s], axis=1)
    size = np.concatenate([np.abs(grad_h * u * s) * (1 + np.abs(g * rest)), np.abs(grad_h * g * s)], axis=1)
    return grad, size
