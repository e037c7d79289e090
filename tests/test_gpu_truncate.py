"""Tokens drawn from truncated distributions and truncated scores through the public entry points, against the plain 64-bit form.  Tokens and what stays are whole
numbers and truth values: they have to be equal (a drawn number or a sum within vocab 2^-(S + 1) of a border, S = min(51, 64 - bits of vocab), where weights in whole numbers may fall on the other side,
does not occur in these draws: 3e-11 of the largest weight at 32,000 scores, 4e-9 at 300,007)."""
import itertools
import math

import numpy as np
import pytest

import paper_2205_10350_amd as ad
from kv8_reference import accept
from truncate_reference import kept, log_prob_tolerance, sample

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

NAN, INF = float("nan"), float("inf")


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def f32(x):
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


def f64(t):
    return t.double().cpu().numpy()


# settings of a row: temperature, k, p, q
SETTINGS = [(1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.3, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.1), (0.8, 50, 0.95, 0.0), (1.0, 300, 0.5, 0.01), (0.2, 0, 0.999, 0.0), (2.5, 1000, 0.8, 0.02),
            (1.0, 1, 0.3, 0.0), (1.0, 0, 0.05, 0.9), (5.0, 0, 0.97, 0.0), (1.0, 700, 1.0, 0.0)]


def settings(rows):
    got = list(itertools.islice(itertools.cycle(SETTINGS), rows))
    return got, dict(zip(("temperature", "top_k", "top_p", "min_p"), (f([g[i] for g in got]) for i, f in enumerate((f32, i32, f32, f32)))))


def as_f32(row):
    return float(np.float32(row[0])), row[1], float(np.float32(row[2])), float(np.float32(row[3]))


def check(x, u, rows, tokens=None, log_probs=None, scores=None):
    """x [rows, vocab] tensor, u numbers, rows: each row's settings."""
    xs = f64(x)
    for r, setting in enumerate(rows):
        setting = as_f32(setting)
        if tokens is not None:
            t, lp = sample(xs[r], u[r], *setting)
            assert int(tokens[r]) == t, (r, setting, int(tokens[r]), t)
            if log_probs is not None:
                got = float(log_probs[r])
                assert (math.isnan(got) and math.isnan(lp)) or abs(got - lp) <= log_prob_tolerance(lp, xs.shape[1]), (r, setting, got, lp)
        if scores is not None:
            stay = kept(xs[r], *setting)
            want = np.where(stay if stay is not None else False, xs[r], -INF)
            assert np.array_equal(f64(scores[r]), want), (r, setting, np.nonzero(f64(scores[r]) != want)[0][:9])


def both(x, u, rows, cut):
    tokens, log_probs = ad.sample_tokens(x, f32(u), log_probs=True, **cut)
    check(x, u, rows, tokens.cpu(), log_probs.cpu(), ad.truncate_scores(x, **cut))
    assert torch.equal(tokens, ad.sample_tokens(x, f32(u), **cut))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 255, 256, 257, 1024, 4095, 4096, 4097, 4099, 8193, 32000, 50021, 70003])
def test_drawn_and_truncated(vocab, bf16):
    n = 3 * len(SETTINGS) if vocab < 9000 else len(SETTINGS)
    rng = np.random.default_rng(vocab)
    x = torch.tensor(rng.standard_normal((n, vocab)) * np.array([1.0, 3.0, 6.0, 0.2])[np.arange(n) % 4, None], dtype=torch.float32)
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    rows, cut = settings(n)
    both(x, rng.random(n).astype(np.float32), rows, cut)


@pytest.mark.parametrize("vocab", [300, 5000, 33000])
def test_equal_scores(vocab):
    """Few different scores, each many times, all equal, zeros of both signs: the indices decide."""
    rng = np.random.default_rng(vocab)
    x = torch.tensor(np.stack([rng.integers(0, 2, vocab), rng.integers(-3, 3, vocab), np.zeros(vocab), rng.integers(0, 400, vocab) / 8, np.where(rng.random(vocab) < 0.5, 0.0, -0.0),
                               np.where(np.arange(vocab) == vocab - 2, 1.0, 0.0)]), dtype=torch.float32)
    x = x.repeat_interleave(len(SETTINGS), 0)
    rows, cut = settings(x.shape[0])
    u = rng.random(x.shape[0]).astype(np.float32)
    both(x.cuda(), u, rows, cut)
    both(x.to(torch.bfloat16).cuda(), u, rows, cut)


def test_numbers_at_the_borders():
    """u and top_p that meet sums exactly (equal scores: sums are whole), the smallest and largest there are."""
    vocab = 4096 + 512
    x = torch.zeros((12, vocab)).cuda()
    u = np.float32([0.0, 0.5, 0.25, 1 - 2.0 ** -24, 2.0 ** -149, 2.0 ** -40, 0.75, 1 / 4608, 0.5, 0.5, 0.0, 0.125])
    p = [1.0, 1.0, 0.5, 1.0, 1.0, 0.5, 0.125, 1.0, 2.0 ** -149, 1 - 2.0 ** -24, 0.0, 0.25]
    rows = [(1.0, 0, q, 0.0) for q in p]
    both(x, u, rows, dict(top_p=f32(p)))


def test_settings_at_their_ends():
    vocab = 5000
    rng = np.random.default_rng(0)
    rows = [(1.0, -5, 1.0, 0.0), (1.0, vocab, 1.0, 0.0), (1.0, vocab + 1, 2.0, -1.0), (1.0, vocab - 1, 1.0, 0.0), (1.0, 2 ** 31 - 1, 1.0, 0.0), (1.0, 0, -1.0, 0.0), (1.0, 0, INF, 0.0),
            (1.0, 0, -INF, 0.0), (1.0, 0, 1.0, 1.0), (1.0, 0, 1.0, 5.0), (1.0, 0, 1.0, 1e-40), (1.0, 0, 0.9, -INF), (1.0, 0, 1.0, INF), (1e-30, 0, 0.9, 0.0), (1e-44, 0, 1.0, 0.0),
            (1e-44, 7, 0.9, 0.5), (1e30, 0, 0.9, 0.0), (3e38, 9, 1.0, 0.5), (0.01, 0, 0.99, 0.0),
            # no distribution
            (0.0, 0, 1.0, 0.0), (-1.0, 0, 1.0, 0.0), (INF, 0, 1.0, 0.0), (NAN, 0, 1.0, 0.0), (1.0, 0, NAN, 0.0), (1.0, 0, 1.0, NAN)]
    n = len(rows)
    x = torch.tensor(rng.standard_normal((n, vocab)) * 3, dtype=torch.float32).cuda()
    cut = dict(zip(("temperature", "top_k", "top_p", "min_p"), (f([g[i] for g in rows]) for i, f in enumerate((f32, i32, f32, f32)))))
    both(x, rng.random(n).astype(np.float32), rows, cut)
    both(x.to(torch.bfloat16), rng.random(n).astype(np.float32), rows, cut)
    # temperatures as large and as small as the scores
    x = torch.tensor(rng.standard_normal((8, vocab)) * np.array([1e38, 1e37, 1e32, 1e30, 1e-30, 1e-36, 1e-38, 1e-40])[:, None], dtype=torch.float32).cuda()
    rows = [(t, 0, p, 0.0) for t, p in zip((3e38, 1e37, 1e32, 5e29, 1e-30, 1e-36, 1e-38, 1e-40), (0.9, 0.99, 1.0, 0.5, 0.9, 0.99, 0.9, 0.6))]
    both(x, rng.random(8).astype(np.float32), rows, dict(temperature=f32([r[0] for r in rows]), top_p=f32([r[2] for r in rows])))


@pytest.mark.parametrize("vocab", [40, 6000])
def test_scores_at_their_ends(vocab):
    """Infinities, NaN, the largest, the smallest and subnormal numbers, rows with nothing or one token left."""
    rng = np.random.default_rng(1)
    base = rng.standard_normal((12, vocab)) * 2
    base[0] = -INF
    base[1] = -INF
    base[1, vocab - 1] = -3.0
    base[2, ::2] = -INF
    base[3, 5] = NAN
    base[4, vocab - 1] = INF
    base[5] *= 1e38
    base[6] *= 1e-42
    base[7, :] = -3.4028234663852886e38
    base[7, 3] = 3.4028234663852886e38
    base[8, 1:] = -INF
    base[9, 0] = NAN
    base[10] = np.where(rng.random(vocab) < 0.9, -INF, base[10])
    x = torch.tensor(base, dtype=torch.float32).repeat_interleave(len(SETTINGS), 0)
    rows, cut = settings(x.shape[0])
    u = rng.random(x.shape[0]).astype(np.float32)
    for some in (x.cuda(), x.to(torch.bfloat16).cuda()):
        both(some, u, rows, cut)


def test_without_settings_and_with_each():
    vocab, n = 9001, 5
    rng = np.random.default_rng(2)
    x = torch.tensor(rng.standard_normal((n, vocab)) * 3, dtype=torch.float32).cuda()
    u = rng.random(n).astype(np.float32)
    both(x, u, [(1.0, 0, 1.0, 0.0)] * n, {})
    for i, (name, value, of) in enumerate((("temperature", 0.6, f32), ("top_k", 40, i32), ("top_p", 0.8, f32), ("min_p", 0.2, f32))):
        row = [1.0, 0, 1.0, 0.0]
        row[i] = value
        both(x, u, [tuple(row)] * n, {name: of([value] * n)})


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_lie_apart_off_alignment_and_in_place(bf16):
    """Views into a wider tensor that begin anywhere, outputs that begin elsewhere, the scores themselves; nothing around them changes."""
    vocab, n = 4500, len(SETTINGS)
    rng = np.random.default_rng(3)
    rows, cut = settings(n)
    u = rng.random(n).astype(np.float32)
    for at, out_at in ((0, 0), (1, 1), (3, 6), (7, 2), (5, 13)):
        wide = torch.tensor(rng.standard_normal((n, vocab + 21)) * 3, dtype=torch.float32)
        wide[:, :at], wide[:, at + vocab:] = NAN, INF
        wide = (wide.to(torch.bfloat16) if bf16 else wide).cuda()
        x = wide[:, at:at + vocab]
        tokens, log_probs = ad.sample_tokens(x, f32(u), log_probs=True, **cut)
        room = torch.full((n, vocab + 30), 7.0, dtype=x.dtype, device="cuda")
        out = ad.truncate_scores(x, out=room[:, out_at:out_at + vocab], **cut)
        check(x, u, rows, tokens.cpu(), log_probs.cpu(), out)
        assert (room[:, :out_at] == 7).all() and (room[:, out_at + vocab:] == 7).all()
        before = wide.clone()
        assert ad.truncate_scores(x, out=x, **cut) is x and torch.equal(x, out)
        assert torch.isnan(wide[:, :at]).all() and (wide[:, at + vocab:] == INF).all() and torch.equal(before[:, :at].isnan(), wide[:, :at].isnan())


@pytest.mark.parametrize("n_seq", [1, 5, 64, 65, 300])
def test_settings_of_sequences(n_seq):
    """Rows looked up in the table: empty sequences, rows before the first and behind the last left as they were."""
    vocab = 700
    rng = np.random.default_rng(n_seq)
    counts = rng.integers(0, 5, n_seq)
    counts[rng.integers(0, n_seq)] = 3
    front, behind = 2, 3
    start = front + np.concatenate(([0], np.cumsum(counts)))
    n = int(start[-1]) + behind
    rows, cut = settings(n_seq)
    x = torch.tensor(rng.standard_normal((n, vocab)) * 3, dtype=torch.float32).cuda()
    u = rng.random(n).astype(np.float32)
    out = torch.full_like(x, 7.0)
    ad.truncate_scores(x, row_start=i32(start), out=out, **cut)
    tokens = ad.sample_tokens(x, f32(u), row_start=i32(start), **cut)
    mine = [rows[b] for b in range(n_seq) for _ in range(counts[b])]
    check(x[front:n - behind], u[front:], mine, tokens[front:n - behind].cpu(), None, out[front:n - behind])
    assert (out[:front] == 7).all() and (out[n - behind:] == 7).all()
    # tables that say something else than there is: nothing is written off the rows
    for wrong in ([-5] * n_seq + [-2], [n] * (n_seq + 1), list(range(n_seq, -1, -1)), [0] * n_seq + [n + 100]):
        ad.truncate_scores(x, row_start=i32(wrong), out=torch.full_like(x, 7.0), **cut)


def test_a_large_vocabulary_and_many_rows():
    rng = np.random.default_rng(4)
    rows, cut = settings(len(SETTINGS))
    x = torch.tensor(rng.standard_normal((len(rows), 300007)) * 2.5, dtype=torch.float32)
    u = rng.random(len(rows)).astype(np.float32)
    both(x.cuda(), u, rows, cut)
    both(x.to(torch.bfloat16).cuda(), u, rows, cut)
    n = 1500
    rows, cut = settings(n)
    x = torch.tensor(rng.standard_normal((n, 600)) * 2.5, dtype=torch.float32).cuda()
    both(x, rng.random(n).astype(np.float32), rows, cut)


def test_a_row_is_the_same_in_every_call():
    rng = np.random.default_rng(5)
    n, vocab = 700, 5000
    rows, cut = settings(n)
    x = torch.tensor(rng.standard_normal((n, vocab)) * 2.5, dtype=torch.float32).cuda()
    u = f32(rng.random(n))
    tokens, log_probs = ad.sample_tokens(x, u, log_probs=True, **cut)
    for lo, hi in ((0, 1), (5, 17), (333, 700)):
        some = {name: t[lo:hi].contiguous() for name, t in cut.items()}
        t, lp = ad.sample_tokens(x[lo:hi], u[lo:hi].contiguous(), log_probs=True, **some)
        assert torch.equal(t, tokens[lo:hi]) and torch.equal(lp, log_probs[lo:hi])
    assert all(torch.equal(a, b) for a, b in zip(ad.sample_tokens(x, u, log_probs=True, **cut), (tokens, log_probs)))


def test_tokens_are_drawn_by_their_probabilities():
    """Evenly spaced numbers draw every token as often as its probability says, to one."""
    rng = np.random.default_rng(6)
    n, vocab = 4096, 50
    one = rng.standard_normal(vocab) * 2
    x = torch.tensor(np.tile(one, (n, 1)), dtype=torch.float32).cuda()
    stay = kept(x[0].double().cpu().numpy(), 1.0, 20, 1.0, 0.0)
    p = np.where(stay, np.exp(x[0].double().cpu().numpy()), 0.0)
    p /= p.sum()
    tokens = ad.sample_tokens(x, f32((np.arange(n) + 0.5) / n), top_k=i32([20] * n))
    assert np.abs(np.bincount(tokens.cpu().numpy(), minlength=vocab) - n * p).max() <= 1.0


def test_captured_and_replayed():
    rng = np.random.default_rng(7)
    n, vocab = len(SETTINGS), 6001
    rows, cut = settings(n)
    x, u = torch.zeros((n, vocab), device="cuda"), torch.zeros(n, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ad.sample_tokens(x, u, log_probs=True, **cut)
        ad.truncate_scores(x, **cut)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tokens, log_probs = ad.sample_tokens(x, u, log_probs=True, **cut)
        scores = ad.truncate_scores(x, **cut)
    for _ in range(4):
        x.copy_(torch.tensor(rng.standard_normal((n, vocab)) * 3, dtype=torch.float32))
        u.copy_(f32(rng.random(n)))
        graph.replay()
        torch.cuda.synchronize()
        check(x, u.cpu().numpy(), rows, tokens.cpu(), log_probs.cpu(), scores)
        assert torch.equal(tokens, ad.sample_tokens(x, u, **cut))


def test_on_another_stream():
    rng = np.random.default_rng(8)
    n, vocab = len(SETTINGS), 6001
    rows, cut = settings(n)
    x, u = torch.tensor(rng.standard_normal((n, vocab)), dtype=torch.float32).cuda(), rng.random(n).astype(np.float32)
    uu, side = f32(u), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tokens, scores = ad.sample_tokens(x, uu, **cut), ad.truncate_scores(x, **cut)
    side.synchronize()
    check(x, u, rows, tokens.cpu(), None, scores)


@pytest.mark.parametrize("bf16", [False, True])
def test_truncated_scores_are_what_sampled_acceptance_takes(bf16):
    """Drafted blocks verified against truncated distributions: tokens that are cut off never stand and are never drawn."""
    rng = np.random.default_rng(9)
    counts, vocab = [8, 0, 3, 25, 1], 5001
    n, start = sum(counts), np.concatenate(([0], np.cumsum(counts)))
    x = torch.tensor(rng.standard_normal((n, vocab)) * 3, dtype=torch.float32)
    x = (x.to(torch.bfloat16) if bf16 else x).cuda()
    rows, cut = settings(len(counts))
    draft = x.float().argmax(-1).to(torch.int32)
    draft[3] = int(x[3].float().argmin())
    u, v = rng.random(n).astype(np.float32) * 0.02, rng.random(len(counts)).astype(np.float32)
    scores = ad.truncate_scores(x, row_start=i32(start), **cut)
    got, tokens = ad.accept_sampled(scores, draft, i32(start), f32(u), f32(v), temperature=cut["temperature"])
    xs = f64(x)
    for b, m in enumerate(counts):
        s = slice(start[b], start[b] + m)
        setting = as_f32(rows[b])
        masked = np.stack([np.where(kept(r, *setting), r, -INF) for r in xs[s]]) if m else xs[s]
        want = accept(masked, draft[s].cpu().numpy(), None, setting[0], u[s], v[b])
        assert got[b].item() == len(want) and tokens[s].tolist() == want + [ad.AD_NEVER] * (m - len(want))
        for i, t in enumerate(want):
            assert masked[i, t] > -INF


def test_refused():
    x = torch.zeros((3, 10), device="cuda")
    u = torch.zeros(3, device="cuda")
    for bad in (dict(u=u[:2]), dict(u=u.double()), dict(u=u.cpu()), dict(temperature=0.8), dict(temperature=u[:2]), dict(top_k=u), dict(top_p=i32([1, 1, 1])), dict(min_p=u.cpu()),
                dict(logits=x.t()), dict(logits=x.half()), dict(row_start=i32([0])), dict(row_start=i32([0, 3]), temperature=u), dict(row_start=[0, 3])):
        a = dict(logits=x, u=u)
        a.update(bad)
        with pytest.raises(ad.AdError) as e:
            ad.sample_tokens(**a)
        assert e.value.code == ad.AD_EINVAL
    for out in (x[:2], x.to(torch.bfloat16), x.cpu(), torch.zeros((10, 3), device="cuda").t(), 3):
        with pytest.raises(ad.AdError):
            ad.truncate_scores(x, out=out)
    wide = torch.zeros((3, 16), device="cuda")
    with pytest.raises(ad.AdError, match="overlap"):
        ad.truncate_scores(wide[:, :10], out=wide[:, 4:14])
    # rows between the scores' rows do not
    fused = torch.randn((3, 2, 10), device="cuda")
    k = i32([2, 3, 1])
    assert torch.equal(ad.truncate_scores(fused[:, 1], top_k=k, out=fused[:, 0]), ad.truncate_scores(fused[:, 1], top_k=k))
    assert torch.equal(ad.truncate_scores(fused[:, 0], top_k=k, out=fused[:, 1]), ad.truncate_scores(fused[:, 0], top_k=k))
    empty = ad.sample_tokens(x[:0], u[:0])
    assert empty.shape == (0,) and ad.truncate_scores(x[:0]).shape == (0, 10)
