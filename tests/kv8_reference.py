"""Plain 64-bit forms (numpy, CPU) of the 8-bit caches, the attention over them and the acceptance of sampled blocks: what the tests of
those operators compare with."""
import math

import numpy as np

BLOCK = 32


def held(x, fmt):
    """What a complete block x [32, width] (float64) stands for; NaN keys of spoiled tokens are the caller's."""
    most = np.abs(x).max()
    if most == 0:
        return x * 0.0
    if fmt == "i8":
        return np.rint(x * 127 / most) * np.float64(np.float32(most) / np.float32(127))
    e = -126
    while most > 448.0 * 2.0 ** e:
        e += 1
    y = x / 2.0 ** e
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -30))), -6) - 3)
    return np.rint(y / step) * step * 2.0 ** e


def tokens_as_read(t, position, fmt, closed=False):
    """t [tokens, heads, width] float64 as a row at `position` reads it: blocks before its own (closed: all) in 8 bits."""
    out = t.copy()
    n = len(t) if closed else min(len(t), position // BLOCK * BLOCK)
    for lo in range(0, n, BLOCK):
        for h in range(t.shape[1]):
            block = np.zeros((BLOCK, t.shape[2]))
            got = t[lo:lo + BLOCK, h]
            block[:len(got)] = got
            out[lo:lo + BLOCK, h] = held(block, fmt)[:len(got)]
    return out


def attend(q, k, v, position, fmt, scale, closed=False):
    """One row q [q_heads, width] over tokens k, v [tokens, heads, width] (growing: those up to `position`).  Returns the output, and for
    every output sum p |v| and sum |q k| scale, what roundings are measured by."""
    if not closed:
        k, v = k[:position + 1], v[:position + 1]
    k, v = tokens_as_read(k, position, fmt, closed), tokens_as_read(v, position, fmt, closed)
    group = q.shape[0] // k.shape[1]
    out, size, dots = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
    for h in range(q.shape[0]):
        kk, vv = k[:, h // group], v[:, h // group]
        if not len(kk):
            continue
        x = kk @ q[h] * scale
        p = np.exp(x - x.max())
        p /= p.sum()
        out[h], size[h], dots[h] = p @ vv, p @ np.abs(vv), (np.abs(kk) @ np.abs(q[h])).max() * abs(scale)
    return out, size, dots


def attend_tolerance(ref, size, dots, width):
    """Roundings on the way: the probabilities to bf16 (2^-8 of each, so of sum p |v|), the result to bf16 (2^-8), and in fp32 the scores: a sum of
    `width` products, one scaling, the exponential's own error (2 steps): (width + 4) 2^-23 of sum |q k| in the exponent, twice (numerator, denominator)."""
    score = 2 * (width + 4) * 2.0 ** -23 * np.maximum(dots, 1.0)
    return 2.0 ** -8 * (np.abs(ref) + size) + size * score + 1e-30


def accept(logits, draft, probs, temperature, u, pick):
    """One sequence's block: the tokens it takes."""
    out = []
    for i in range(len(draft)):
        x = logits[i].astype(np.float64)
        if not (0 < temperature < math.inf) or np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any():
            return out
        x = x / np.float64(temperature)
        p = np.exp(x - x.max())
        p /= p.sum()
        d = int(draft[i])
        q = np.zeros_like(p)
        if 0 <= d < len(p):
            if probs is None:
                q[d] = 1.0
            else:
                q = probs[i].astype(np.float64)
            if np.float64(u[i]) * q[d] < p[d]:
                out.append(d)
                continue
        r = np.where(np.arange(len(p)) == d, 0.0, p) if probs is None else np.maximum(p - q, 0.0)
        c = np.cumsum(r)
        hit = np.nonzero(c > np.float64(pick) * c[-1])[0]
        out.append(int(hit[0]) if len(hit) else int(np.nonzero(r)[0][-1]) if r.any() else d)
        break
    return out
