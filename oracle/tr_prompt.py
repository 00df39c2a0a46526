"""CPU oracle of rotary positions, causal attention of chunks and sampled tokens (numpy, 64 bits, one
sequence or row at a time).  Written from the rules in include/trjacobi.h; test infrastructure only."""
import math

import numpy as np


def depths(parent):
    d = np.zeros(len(parent), int)
    for i in range(1, len(parent)):
        d[i] = d[parent[i]] + 1
    return d


def rotary_freqs(rot, theta, scaling="plain", factor=1.0, low=1.0, high=4.0, trained=1):
    """Frequencies of all pairs and what rotated rows are multiplied by."""
    out, mag = np.zeros(rot // 2), 1.0
    pair = lambda turns: rot * math.log(trained / (2 * math.pi * turns)) / (2 * math.log(theta))  # noqa: E731
    for j in range(rot // 2):
        f = theta ** (-2.0 * j / rot)
        if scaling == "linear":
            f = f / factor
        elif scaling == "turns":
            t = trained * f / (2 * math.pi)
            if t <= low:
                f = f / factor
            elif t < high:
                g = (t - low) / (high - low)
                f = f / factor * (1 - g) + f * g
        elif scaling == "ramp":
            a, z = max(0, math.floor(pair(high))), min(rot - 1, math.ceil(pair(low)))
            z = z if z != a else a + 0.001
            r = min(1.0, max(0.0, (j - a) / (z - a)))
            f = f * (1 - r) + f / factor * r
            mag = 0.1 * math.log(factor) + 1
        out[j] = f
    return out, mag


def rotary(x, positions, freqs, magnitude, pairs):
    """x [n, heads, dh] at positions [n]."""
    half = len(freqs)
    y = x.astype(np.float64).copy()
    for i, p in enumerate(positions):
        for j in range(half):
            c1, c2 = (2 * j, 2 * j + 1) if pairs else (j, j + half)
            c, s = math.cos(int(p) * float(freqs[j])), math.sin(int(p) * float(freqs[j]))
            x1, x2 = x[i, :, c1].astype(np.float64), x[i, :, c2].astype(np.float64)
            y[i, :, c1] = magnitude * (x1 * c - x2 * s)
            y[i, :, c2] = magnitude * (x1 * s + x2 * c)
    return y


def chunk_attention(q, keys, values, k_rows, v_rows, scale):
    """One sequence: q [n, H, dh], keys and values [Hkv, L, dh] of the cache, rows [n, Hkv, dh]: row i sees the
    cache and rows 0 .. i.  Returns the result and the same weights' mean of |v|."""
    n, H, dh = q.shape
    L, group = keys.shape[1], H // keys.shape[0]
    hidden = np.arange(L + n)[None] > L + np.arange(n)[:, None]
    out, mean = np.zeros((n, H, dh)), np.zeros((n, H, dh))
    for h in range(H):
        k = np.concatenate([keys[h // group], k_rows[:, h // group]]).astype(np.float64)
        v = np.concatenate([values[h // group], v_rows[:, h // group]]).astype(np.float64)
        score = scale * (q[:, h].astype(np.float64) @ k.T)
        score[hidden] = -np.inf
        w = np.exp(score - score.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        out[:, h], mean[:, h] = w @ v, w @ np.abs(v)
    return out, mean


UNIT = 2 ** 38


def order(x):
    """Indices of the tokens of a row, larger first, of equal ones the lowest index first."""
    some = [i for i in range(len(x)) if x[i] > -np.inf]
    return sorted(some, key=lambda i: (-float(x[i]), i))


def weights(x, picked, t):
    top = float(x[picked[0]])
    return [UNIT if float(x[i]) == top else 0 if math.isinf(top) else
            int(np.rint(np.exp((float(x[i]) - top) / float(t)) * UNIT)) for i in picked]


def kept(x, rules):
    """Tokens that the rules keep, in order, and their weights as whole numbers."""
    t, k, p, m = (float(r) for r in rules)
    some = order(x)
    if not some:
        return [], []
    if t == 0:
        return some[:1], [UNIT]
    if k >= 1:
        some = some[:int(min(k, len(some)))]
    w = weights(x, some, t)
    if p < 1:
        need, run, n = math.ceil(max(p, 0.0) * float(sum(w))), 0, 0
        while n == 0 or run < need:
            run += w[n]
            n += 1
        some, w = some[:n], w[:n]
    least = math.ceil(min(max(m, 0.0), 1.0) * UNIT)
    n = sum(v >= least for v in w)
    return some[:n], w[:n]


def sample(x, rules, u):
    """Token of a row and its probability; -1 and 0 where there is no token."""
    some, w = kept(x, rules)
    if not some:
        return -1, 0.0
    u = 0.0 if u != u else min(max(float(u), 0.0), 1 - 2.0 ** -24)
    target, run = min(math.floor(u * float(sum(w))), sum(w) - 1), 0
    for i, v in zip(some, w):
        run += v
        if run > target:
            return i, v / sum(w)
    raise AssertionError("the running sum ends above every target")
