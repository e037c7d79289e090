"""Truncated distributions where a row's many small weights matter: temperatures far below the scores' differences."""
import numpy as np
import pytest

import paper_2205_10350_amd as ad
from truncate_reference import kept, log_prob_tolerance, sample

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

INF = float("inf")


def f32(x):
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


def check(x, u, rows):
    """Tokens, logarithms of their probabilities and truncated scores of x [rows, vocab]; rows: each row's (T, k, p, q)."""
    cut = dict(zip(("temperature", "top_k", "top_p", "min_p"), (f32([r[0] for r in rows]), torch.tensor([r[1] for r in rows], dtype=torch.int32, device="cuda"), f32([r[2] for r in rows]),
                                                                f32([r[3] for r in rows]))))
    tokens, log_probs = ad.sample_tokens(x, f32(u), log_probs=True, **cut)
    scores = ad.truncate_scores(x, **cut).double().cpu().numpy()
    xs = x.double().cpu().numpy()
    for r, (t, k, p, q) in enumerate(rows):
        setting = float(np.float32(t)), k, float(np.float32(p)), float(np.float32(q))
        want, lp = sample(xs[r], float(np.float32(u[r])), *setting)
        assert int(tokens[r]) == want, (r, setting, int(tokens[r]), want)
        assert abs(float(log_probs[r]) - lp) <= log_prob_tolerance(lp, x.shape[1]), (r, setting, float(log_probs[r]), lp)
        stay = kept(xs[r], *setting)
        assert np.array_equal(scores[r], np.where(stay, xs[r], -INF)), (r, setting, int((scores[r] > -INF).sum()), int(stay.sum()))


@pytest.mark.parametrize("vocab,near", [(3000, 7), (3000, 200), (5000, 2500), (33000, 100), (33000, 20000)])
def test_temperatures_far_below_the_scores(vocab, near):
    """`near` tokens within 8 T of the largest, all others hundreds to millions of T below it: they weigh nothing, however small T is."""
    rng = np.random.default_rng(vocab + near)
    x, rows = [], []
    for t, lo, hi in ((1e-36, 750, 1e6), (1e-30, 750, 2000), (1e-33, 900, 1e6), (1e-37, 1e3, 2e10), (1e-44, 1e3, 1e6), (1e-30, 1e5, 1e9), (2e-29, 100, 4000)):
        t = float(np.float32(t))
        for p in (0.5, 0.9, 0.999, 1.0):
            row = -t * np.exp(rng.uniform(np.log(lo), np.log(hi), vocab))
            row[rng.permutation(vocab)[:near]] = -t * rng.uniform(0, 8, near)
            x.append(row)
            rows.append((t, 0, p, 0.0))
        rows[-2] = (t, 40, 0.9, 0.0)
    check(f32(np.stack(x)), rng.random(len(rows)).astype(np.float32), rows)
