"""Plain 64-bit forms (numpy, CPU) of truncated distributions: what the tests of those operators compare with."""
import math

import numpy as np


def weights(x, temperature):
    """exp((x - max x) / T), float64; None: no distribution."""
    x = np.asarray(x, np.float64)
    if not (0 < temperature < math.inf) or np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
        return None
    with np.errstate(over="ignore"):
        return np.exp((x - x.max()) / np.float64(temperature))


def kept(x, temperature=1.0, k=0, p=1.0, q=0.0):
    """Which tokens stay: truth values; None: no distribution."""
    w = weights(x, temperature)
    if w is None or math.isnan(p) or math.isnan(q):
        return None
    x = np.asarray(x, np.float64)
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if 0 < k < len(x):
        order = order[:k]
    if p < 1:
        sums = np.cumsum(w[order])
        enough = np.nonzero(sums >= np.float64(p) * sums[-1])[0]
        order = order[:max(int(enough[0]), 0) + 1]
    out = np.zeros(len(x), bool)
    out[order] = True
    return out & (w >= min(np.float64(q), 1.0))


def sample(x, u, temperature=1.0, k=0, p=1.0, q=0.0):
    """(token, logarithm of its probability among those that stay); (-1, NaN) without a distribution."""
    stay = kept(x, temperature, k, p, q)
    if stay is None:
        return -1, math.nan
    w = np.where(stay, weights(x, temperature), 0.0)
    sums = np.cumsum(w)
    t = int(np.nonzero(sums > np.float64(u) * sums[-1])[0][0])
    x = np.asarray(x, np.float64)
    return t, (x[t] - x.max()) / np.float64(temperature) - math.log(w.sum())


def log_prob_tolerance(value, vocab):
    """The fp32 result's rounding, 2^-24 of it; weights are whole numbers of 2^-S of the largest, S = min(51, 64 - bits of vocab), each off by half at most, which beside a sum of
    1 or more moves its logarithm by vocab 2^-(S + 1): an eighth of the second number here (up to 2^13 scores: half of it at most); the rest (exponentials to 3.3e-13, a logarithm, three additions of numbers below 2^6,
    as a drawn token weighs a unit or more) is below 2^-41, half of the third."""
    return 2.0 ** -24 * abs(value) + vocab * 2.0 ** -min(51, 62 - vocab.bit_length()) + 2.0 ** -40
