"""The oracle's decoder with its keys and values as caches in 8 bits hold them, models whose attention is peaked (so that keys, scales and
blocks matter to the scores), and the ways in which such a decoder could be wrong."""
import numpy as np

from ad_inputs import SPECIAL, init_weights, model_dims
from kv8_reference import BLOCK, tokens_as_read
from oracle import ad_oracle as O

S, T = 70, 130     # source and output tokens: three blocks of memory, four complete blocks of the decoder's own cache
# format; what is added to every 32nd bias of the keys; factor of the decoder's query and key matrices; seed
# An outlier among a key's columns leaves the softmax as it is (the same for every key), but a block's scale goes by it: 8-bit steps become
# large beside the other columns, and a cache that is not held in 8 bits shows.
MODELS = [("e4m3", 200, 5, 23), ("i8", 0, 7, 23), ("i8", 200, 3, 23)]
WRONG = ["zero keys", "zero values", "first block", "own block", "scale", "unquantised"]


class HeldOracle(O.Model):
    """`wrong`: (what is wrong, of the closed caches or of the growing ones)."""
    fmt, deciding, wrong = "e4m3", False, None

    def decode_full(self, memory, tokens, causal=True):
        self.deciding = True
        try:
            return super().decode_full(memory, tokens, causal)
        finally:
            self.deciding = False

    def attention(self, q, k, v, vis):
        if not self.deciding:
            return super().attention(q, k, v, vis)
        closed = vis[0] == vis[-1] and len(vis) > 1
        what = self.wrong[0] if self.wrong and self.wrong[1] == closed else None
        heads = lambda t: O.bf16_round(t).reshape(len(t), self.H, self.dh)
        k, v = heads(k), heads(v)
        if what == "zero keys":
            k = np.zeros_like(k)
        if what == "zero values":
            v = np.zeros_like(v)
        out = []
        for i in range(len(q)):
            n, lo = vis[i], 0
            if what == "first block":
                n = min(n, BLOCK)
            if what == "own block" and not closed:
                lo = i // BLOCK * BLOCK
            kk, vv = (t[:n] if what == "unquantised" else tokens_as_read(t[:n], i, self.fmt, closed) for t in (k, v))
            if what == "scale" and n > BLOCK:       # one head's first block of keys
                kk = kk.copy()
                kk[:BLOCK, 0] *= 2
            out.append(super().attention(q[i:i + 1], kk[lo:].reshape(-1, self.d), vv[lo:].reshape(-1, self.d), [n - lo])[0])
        return np.stack(out)


def problem(fmt, outlier, factor, seed):
    """dims, weights, source, tokens"""
    dims = model_dims("tiny")
    w = init_weights(dims, seed, 0.02)
    for n in w:
        if n.startswith("dec") and (".self.w" in n or ".cross.w" in n):
            w[n] = w[n] * np.float32(factor if n[-1] in "qk" else 5)
        if n.startswith("dec") and n.endswith(".bk"):
            w[n][::32] = outlier
    rng = np.random.default_rng(seed)
    return dims, w, rng.integers(5, dims["vocab"], size=S).astype(np.int32), rng.integers(5, dims["vocab"], size=T).tolist()


def scores(fmt, dims, w, src, tok, contract=True, wrong=None):
    """Of all rows; contract: with the bf16 path's rounding points."""
    m = HeldOracle(dims, {n: (O.bf16_round(a) if a.ndim == 2 else a) for n, a in w.items()}, np.float64, contract=contract, max_pos=256)
    m.fmt, m.wrong = fmt, wrong
    return m.decode_full(m.encode(src), [SPECIAL["bos"]] + tok[:-1])


def far(a, b):
    """The median over the rows that read 8-bit blocks of their own cache of the scores' rms difference (a rounding that falls the other way moves a held value by a whole
    step, and single rows by many times the others: the median does not go by them)."""
    return float(np.median(np.sqrt(((a - b)[BLOCK:] ** 2).mean(1))))


def tolerance(fmt, dims, w, src, tok):
    """(scores with the bf16 roundings, how far from them the device's may be).  The device rounds at the same points, its 32-bit sums then let some roundings fall the
    other way.  That cannot be more than roundings at these points do altogether, which is what lies between the scores with and without them; half as much again for the spread of such a number
    from one draw of the roundings to another."""
    want = scores(fmt, dims, w, src, tok)
    return want, 1.5 * far(want, scores(fmt, dims, w, src, tok, contract=False))
