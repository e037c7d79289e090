"""Sequences of 8-bit caches copied, and attention over texts that sequences share, through the public entry points: copies bit for bit, attention against the plain 64-bit form."""
import numpy as np
import pytest

import paper_2205_10350_amd as ad
from kv8_reference import attend_tolerance, tokens_as_read
from truncate_reference import sample

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

NAN, INF = float("nan"), float("inf")


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def starts(n):
    return i32(np.concatenate(([0], np.cumsum(n))))


def draw(seed, *shape, spread=0.5):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal((1,) * (len(shape) - 1) + shape[-1:]))
    return torch.tensor(x, dtype=torch.float32).to(torch.bfloat16)


def f64(t):
    return t.double().cpu().numpy()


def packed(t, at, n):
    return torch.cat([t[b, a:a + m] for b, (a, m) in enumerate(zip(at, n)) if m]).cuda()


def stale(cache):
    """Whatever lies in the memory must not matter: NaN patterns of every type."""
    cache.memory.fill_(0xFF)
    return cache


def feed(cache, k, v, lens, step):
    for at in range(0, max(lens), step):
        part = [max(0, min(n - at, step)) for n in lens]
        begin = [min(at, n) for n in lens]
        cache.append(packed(k, begin, part), packed(v, begin, part), starts(part), i32(begin))


def read(cache, b, begin, end):
    """Tokens begin .. end - 1 of sequence b as the row behind them reads them, fp32."""
    n = [end - begin if i == b else 0 for i in range(cache.cfg.n_seq)]
    return torch.stack(cache.read(starts(n), i32([begin] * len(n)), i32([end] * len(n)), rows=end - begin, dtype=torch.float32))


def same(a, b):
    return torch.equal(a.view(torch.int32), b.view(torch.int32))


# ---- copies ----------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("closed", [False, True])
@pytest.mark.parametrize("fmt,width,heads", [("e4m3", 64, 2), ("i8", 32, 3), ("e4m3", 128, 1)])
def test_forked_within_a_cache(fmt, width, heads, closed):
    """Each length to another place: the copy reads as its source, and so it does with what is appended to both."""
    lens = [1, 31, 32, 33, 64, 95, 100, 5]
    n = len(lens)
    k, v = draw(1, n, 140, heads, width), draw(2, n, 140, heads, width)
    cache = stale(ad.Kv8Cache(2 * n + 1, heads, width, capacity=140, k_max=40, format=fmt, closed=closed))
    feed(cache, k, v, lens + [0] * (n + 1), 140 if closed else 40)
    before = [read(cache, b, 0, m) for b, m in enumerate(lens)]
    places = [n + 1 + i for i in range(n)]
    cache.copy(i32(range(n)), i32(places), i32(lens))
    for b, m in enumerate(lens):
        assert same(read(cache, places[b], 0, m), before[b]) and same(read(cache, b, 0, m), before[b]), b
    if closed:
        q = draw(3, 2 * n + 1, heads, width).cuda()
        q[places[0]:] = q[:n]
        out = cache.attend(q, i32(list(range(2 * n + 2))), i32(lens + [0] + lens))
        assert torch.equal(out[:n], out[n + 1:])
        return
    rows = [20] * n + [0] + [20] * n
    both = lens + [0] + lens
    kk, vv = (torch.cat((packed(t, lens, [20] * n),) * 2) for t in (k, v))
    cache.append(kk, vv, starts(rows), i32(both))
    for b, m in enumerate(lens):
        assert same(read(cache, places[b], 0, m + 20), read(cache, b, 0, m + 20)), b
    q = torch.cat((draw(4, 20 * n, heads, width),) * 2).cuda()
    out = cache.attend(q, starts(rows), i32(both))
    assert torch.equal(out[:20 * n], out[20 * n:]) and torch.isfinite(out).all()


@pytest.mark.parametrize("n", [1, 2, 7, 40, 300])
def test_all_are_read_before_any_is_written(n):
    """Permutations, shifts by one, cycles, many copies of one, places that are themselves sources: as gathered at once."""
    heads, width, most = (4, 64, 100) if n < 100 else (1, 32, 70)
    rng = np.random.default_rng(n)
    lens = rng.integers(1, most + 1, n).tolist()
    k, v = draw(5, n, most, heads, width), draw(6, n, most, heads, width)
    cache = stale(ad.Kv8Cache(n, heads, width, capacity=most, k_max=most))
    feed(cache, k, v, lens, most)
    for how in (rng.permutation(n), np.roll(np.arange(n), 1), np.roll(np.arange(n), -1), np.arange(n)[::-1], np.full(n, n // 2), rng.integers(0, n, n), np.arange(n)):
        want = [read(cache, int(b), 0, lens[b]) for b in how]
        order = rng.permutation(n)                        # (entries in any order)
        cache.copy(i32(how[order]), i32(order), i32([lens[how[i]] for i in order]), max_tokens=most if n % 2 else None)
        lens = [lens[b] for b in how]
        for b in range(n):
            assert same(read(cache, b, 0, lens[b]), want[b]), (how, b)


def test_moved_together_in_a_large_cache():
    """The gaps of sequences that ended are closed, every sequence moved one place or more, over many blocks and heads."""
    heads, width, most, n = 16, 64, 1500, 24
    k, v = draw(7, n, most, heads, width), draw(8, n, most, heads, width)
    lens = np.random.default_rng(9).integers(1, most, n).tolist()
    cache = stale(ad.Kv8Cache(n, heads, width, capacity=most, k_max=most, format="i8"))
    feed(cache, k, v, lens, most)
    stay = [b for b in range(n) if b % 5 != 0]
    want = [read(cache, b, 0, lens[b]) for b in stay]
    cache.copy(i32(stay), i32(range(len(stay))), i32([lens[b] for b in stay]))
    for i, b in enumerate(stay):
        assert same(read(cache, i, 0, lens[b]), want[i]), b


@pytest.mark.parametrize("closed", [False, True])
def test_taken_over_from_another_cache(closed):
    """Other sizes of the cache, other rings, from a block on."""
    heads, width, fmt = 2, 64, "e4m3"
    lens = [200, 33, 64, 97, 180, 31]
    n = len(lens)
    k, v = draw(10, n, 240, heads, width), draw(11, n, 240, heads, width)
    origin = stale(ad.Kv8Cache(n, heads, width, capacity=240, k_max=100, format=fmt, closed=closed))
    feed(origin, k, v, lens, 240 if closed else 100)
    cache = stale(ad.Kv8Cache(9, heads, width, capacity=230, k_max=7, format=fmt, closed=closed))
    begin = [96, 0, 32, 64, 160, 0]
    places = [8, 0, 3, 4, 1, 7]
    cache.copy(i32(range(n)), i32(places), i32(lens), begin=i32(begin), origin=origin, max_tokens=230)
    for b in range(n):
        assert same(read(cache, places[b], 0, lens[b] - begin[b]), read(origin, b, begin[b], lens[b])), b
    if not closed:                                        # what follows: as if all of it had been written there
        other = stale(ad.Kv8Cache(9, heads, width, capacity=230, k_max=7, format=fmt))
        k2, v2 = (torch.zeros((9, 240, heads, width), dtype=torch.bfloat16) for _ in range(2))
        have = [0] * 9
        for b in range(n):
            have[places[b]] = lens[b] - begin[b]
            for t2, t in ((k2, k), (v2, v)):
                t2[places[b], :240 - begin[b]] = t[b, begin[b]:]
        feed(other, k2, v2, have, 7)
        q = draw(12, 7 * n, heads, width).cuda()
        rows = [7 if h else 0 for h in have]
        got = []
        for c in (cache, other):
            c.append(packed(k2, have, rows), packed(v2, have, rows), starts(rows), i32(have))
            got.append(c.attend(q, starts(rows), i32(have)))
        assert torch.equal(*got)


def test_shorter_than_the_source():
    """A source that is copied up to a token it may be taken back to."""
    heads, width = 2, 32
    k, v = draw(13, 1, 90, heads, width), draw(14, 1, 90, heads, width)
    for end in (32, 64, 65, 70, 80, 90, 1):
        cache = stale(ad.Kv8Cache(3, heads, width, capacity=90, k_max=90))
        cache.append(k[0].cuda(), v[0].cuda(), starts([90, 0, 0]), i32([0, 0, 0]))
        cache.copy(i32([0]), i32([2]), i32([end]))
        for g, t in zip(read(cache, 2, 0, end), (k, v)):
            assert torch.equal(g.cpu(), torch.tensor(tokens_as_read(f64(t[0, :end]), end, "e4m3")).float()), end


def test_entries_are_held_to_the_caches():
    """Sequences, lengths and places that are not there, and places given twice: the first entry counts, nothing else changes."""
    heads, width, n, most = 2, 32, 4, 70
    k, v = draw(15, n, most, heads, width), draw(16, n, most, heads, width)
    lens = [70, 40, 33, 5]
    cache = stale(ad.Kv8Cache(n, heads, width, capacity=most, k_max=most))
    feed(cache, k, v, lens, most)
    before = cache.memory.clone()
    for source, place, end in (([-1, 4, 100, 2 ** 31 - 1], [0, 1, 2, 3], [70] * 4), ([0, 1, 2, 3], [-1, 4, 2 ** 31 - 1, -2 ** 31], [70] * 4), ([0, 1, 2, 3], [3, 2, 1, 0], [0, -1, -70, -2 ** 31]),
                               ([], [], [])):
        cache.copy(i32(source), i32(place), i32(end))
        assert torch.equal(cache.memory, before), source
    was = [read(cache, b, 0, m) for b, m in enumerate(lens)]
    cache.copy(i32([9, 1, 2, 0]), i32([3, 3, 3, 3]), i32([70, 40, 33, 70]))
    assert same(read(cache, 3, 0, 40), was[1])
    cache.copy(i32([0]), i32([2]), i32([1000]))                                           # (no more than the capacity)
    assert same(read(cache, 2, 0, 70), was[0]) and same(read(cache, 0, 0, 70), was[0])
    small = stale(ad.Kv8Cache(1, heads, width, capacity=64, k_max=3))
    small.copy(i32([0]), i32([0]), i32([70]), origin=cache)                               # (nor of the other)
    assert same(read(small, 0, 0, 64), was[0][:, :64])
    small.copy(i32([0]), i32([0]), i32([70]), begin=i32([-40]), origin=cache)
    small.copy(i32([0]), i32([0]), i32([70]), begin=i32([96]), origin=cache)              # (begins behind its end)
    assert same(read(small, 0, 0, 64), was[0][:, :64])


def test_copies_are_refused():
    make = lambda **kw: ad.Kv8Cache(**dict(dict(n_seq=2, n_heads=2, head_width=32, capacity=64, k_max=4), **kw))  # noqa: E731
    cache, one = make(), i32([0])
    for kw in (dict(begin=one), dict(origin=make(n_heads=1)), dict(origin=make(head_width=64)), dict(origin=make(format="i8")), dict(origin=make(closed=True)), dict(origin=3),
               dict(max_tokens=-1), dict(source=i32([0, 1])), dict(source=one.long()), dict(place=one.cpu()), dict(end=[3]), dict(source=i32([[0]])),
               dict(source=i32([0, 1, 1]), place=i32([0, 1, 1]), end=i32([1, 1, 1]))):
        a = dict(source=one, place=one, end=one)
        a.update(kw)
        with pytest.raises(ad.AdError) as e:
            cache.copy(**a)
        assert e.value.code == ad.AD_EINVAL, kw
    cache.copy(one, one, one, origin=cache)                                               # (itself)


def test_a_copy_past_32_bits():
    heads, width, cap, n = 8, 128, 1 << 17, 17
    cache = ad.Kv8Cache(n, heads, width, capacity=cap, k_max=64)
    k, v = draw(17, 1, 70, heads, width), draw(18, 1, 70, heads, width)
    base = cap - 96
    for lo, m in ((0, 64), (64, 6)):
        cache.append(k[0, lo:lo + m].cuda(), v[0, lo:lo + m].cuda(), starts([0] * (n - 2) + [m, 0]), i32([0] * (n - 2) + [base + lo, 0]))
    cache.copy(i32([n - 2]), i32([n - 1]), i32([base + 70]))
    assert same(read(cache, n - 1, base, base + 70), read(cache, n - 2, base, base + 70))
    for g, t in zip(read(cache, n - 1, base, base + 70), (k, v)):
        assert torch.equal(g.cpu(), torch.tensor(tokens_as_read(f64(t[0]), 70, "e4m3")).float())


# ---- shared texts --------------------------------------------------------------------------------------------------------------------------
def reference(q, text, own, position, fmt, scale):
    """One row q [q_heads, width] over a text (k, v) in 8 bits throughout and the tokens (k, v) of its own sequence up to `position`; with what roundings are measured by."""
    k, v = (np.concatenate((tokens_as_read(t, 0, fmt, True), tokens_as_read(o[:position + 1], position, fmt))) for t, o in zip(text, own))
    group = q.shape[0] // k.shape[1]
    out, size, dots = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
    for h in range(q.shape[0]):
        kk, vv = k[:, h // group], v[:, h // group]
        x = kk @ q[h] * scale
        p = np.exp(x - x.max())
        p /= p.sum()
        out[h], size[h], dots[h] = p @ vv, p @ np.abs(vv), (np.abs(kk) @ np.abs(q[h])).max() * abs(scale)
    return out, size, dots


class Problem:
    def __init__(self, fmt, width, heads, q_heads, each, text, lens, rows, closed, seed=20, capacity=None, k_max=None):
        n = len(lens)
        self.fmt, self.each, self.text, self.lens, self.rows = fmt, each, text, lens, rows
        self.tk, self.tv = draw(seed, len(text), max(text + [1]), heads, width), draw(seed + 1, len(text), max(text + [1]), heads, width)
        most = max(a + m for a, m in zip(lens, rows))
        self.k, self.v, self.q = draw(seed + 2, n, most, heads, width), draw(seed + 3, n, most, heads, width), draw(seed + 4, sum(rows), q_heads, width)
        self.shared = stale(ad.Kv8Cache(len(text), heads, width, capacity=max(text + [1]) if capacity is None else capacity, k_max=90, format=fmt, closed=closed))
        feed(self.shared, self.tk, self.tv, text, max(text + [1]) if closed else 90)
        step = max(rows + [1])
        self.cache = stale(ad.Kv8Cache(n, heads, width, capacity=most + 3, k_max=step if k_max is None else k_max, format=fmt))
        feed(self.cache, self.k, self.v, lens, step)
        self.cache.append(packed(self.k, lens, rows), packed(self.v, lens, rows), starts(rows), i32(lens))
        self.first = [0] + np.cumsum(each).tolist()

    def go(self, **kw):
        a = dict(q=self.q.cuda(), row_start=starts(self.rows), length=i32(self.lens), shared=self.shared, seq_start=i32(self.first), shared_length=i32(self.text))
        a.update(kw)
        return self.cache.attend_shared(**a)

    def owner(self, b):
        return next((g for g in range(len(self.text)) if self.first[g] <= b < self.first[g + 1]), None)

    def want(self, r, b, i, scale=None):
        g = self.owner(b)
        text = [f64(t[g, :self.text[g]]) if g is not None else f64(t[0, :0]) for t in (self.tk, self.tv)]
        return reference(f64(self.q[r]), text, [f64(t[b]) for t in (self.k, self.v)], self.lens[b] + i, self.fmt, self.q.shape[2] ** -0.5 if scale is None else scale)

    def check(self, got, every=1, scale=None):
        got = f64(got)
        r = 0
        for b, m in enumerate(self.rows):
            for i in range(m):
                if r % every == 0:
                    ref, size, dots = self.want(r, b, i, scale)
                    tol = attend_tolerance(ref, size, dots, self.q.shape[2])
                    assert np.all(np.abs(got[r] - ref) <= tol), (b, i, np.max(np.abs(got[r] - ref) / tol))
                r += 1


# (query heads that share a head, the texts' capacity) of all in one launch, of workgroups of 32 rows and of 128
FORMS = [(1, None), (1, 1100), (32, None)]

CASES = [
    # format, width, heads, query heads, sequences of each text, lengths of the texts, own tokens, rows, closed
    ("e4m3", 64, 2, 2, [3, 1], [64, 96], [0, 1, 40, 33], [1, 1, 1, 1], False),
    ("i8", 64, 2, 2, [2, 0, 3], [700, 5, 33], [0, 31, 32, 100, 7], [25, 1, 9, 3, 40], True),
    ("i8", 64, 2, 2, [2, 0, 3], [1700, 5, 33], [0, 31, 32, 100, 7], [25, 1, 9, 3, 40], True),
    ("e4m3", 32, 3, 6, [1, 4], [1, 1030], [5, 600, 0, 64, 2], [33, 1, 2, 1, 70], True),
    ("i8", 32, 1, 1, [6], [1600], [1, 2, 3, 4, 5, 6], [8] * 6, False),
    ("e4m3", 128, 1, 4, [2, 2], [520, 0], [3, 30, 0, 77], [1, 2, 5, 1], True),
    ("i8", 128, 2, 10, [3], [1056], [40, 0, 600], [2, 7, 1], False),
    ("e4m3", 64, 1, 16, [1, 1], [2112, 32], [0, 0], [3, 1], False),
    ("e4m3", 64, 1, 2, [40], [544], list(range(40)), [1] * 39 + [5], False),
    # (64 or more rows of a head to a text: workgroups of 128 rows)
    ("i8", 128, 1, 16, [6, 5], [1300, 40], [0, 70, 3, 31, 32, 33, 5, 9, 64, 1, 100], [1, 2, 9, 1, 3, 1, 1, 20, 1, 1, 4], True),
    ("e4m3", 128, 2, 32, [5], [2144], [7, 0, 40, 1, 90], [3, 1, 1, 8, 1], False),
    ("e4m3", 32, 2, 64, [1, 0, 5], [33, 64, 3001], [0, 9, 31, 500, 2, 64], [2, 1, 3, 1, 1, 5], True),
    ("i8", 32, 1, 64, [2, 1], [1088, 0], [0, 35, 8], [5, 1, 2], False),
    ("i8", 64, 2, 128, [2, 1], [1500, 31], [0, 35, 8], [3, 1, 2], True),
]


@pytest.mark.parametrize("case", CASES)
def test_attention_over_shared_texts(case):
    p = Problem(*case)
    got = p.go()
    p.check(got)
    rows = [sum(p.rows[a:b]) for a, b in zip(p.first, p.first[1:])]
    most = max(a + m for a, m in zip(p.lens, p.rows))
    assert torch.equal(got, p.go(max_rows=max(p.rows), max_keys=most, max_shared_rows=max(rows), max_shared_keys=max(p.text)))
    # the same bits alone: one sequence at a time, the others without rows
    r = 0
    for b, m in enumerate(p.rows):
        if b % 3 == 0 or m > 20:
            one = [m if i == b else 0 for i in range(len(p.rows))]
            assert torch.equal(got[r:r + m], p.go(q=p.q[r:r + m].cuda(), row_start=starts(one), max_rows=m)), b
            last = [1 if i == b else 0 for i in range(len(p.rows))]
            at = [n + m - 1 if i == b else n for i, n in enumerate(p.lens)]
            assert torch.equal(got[r + m - 1:r + m], p.go(q=p.q[r + m - 1:r + m].cuda(), row_start=starts(last), length=i32(at))), b
        r += m


@pytest.mark.parametrize("group,capacity", FORMS)
@pytest.mark.parametrize("closed", [False, True])
def test_sequences_of_no_text_texts_of_no_sequence_and_empty_texts(closed, group, capacity):
    text = [64, 32, 0, 96]
    p = Problem("e4m3", 64, 2, 2 * max(group, 2), [0, 2, 1, 1], text, [10, 20, 0, 33, 5, 40], [2, 1, 3, 1, 1, 2], closed, capacity=capacity)
    p.first = [1, 1, 3, 4, 5]                  # sequences 0 and 5 of no text, text 0 of none, text 2 empty
    got = p.go()
    p.check(got)
    alone = p.cache.attend(p.q.cuda(), starts(p.rows), i32(p.lens))
    r = np.cumsum([0] + p.rows)
    for b in (0, 3, 5):
        assert torch.equal(got[r[b]:r[b + 1]], alone[r[b]:r[b + 1]])
    assert torch.equal(p.go(max_shared_keys=0), alone) and not torch.equal(got, alone)


def test_the_text_in_the_same_cache():
    """Forks within one cache: the first sequence is the text of the others, whose own tokens are the ones behind its whole blocks."""
    heads, width, n, text = 2, 64, 5, 150
    whole = text // 32 * 32
    cache = stale(ad.Kv8Cache(n, heads, width, capacity=300, k_max=150))
    k, v = draw(30, n, 300, heads, width), draw(31, n, 300, heads, width)
    k[1:, :text], v[1:, :text] = k[:1, :text], v[:1, :text]
    feed(cache, k, v, [text] + [0] * (n - 1), 150)
    origin = stale(ad.Kv8Cache(1, heads, width, capacity=300, k_max=150))
    feed(origin, k[:1], v[:1], [text], 150)
    cache.copy(i32([0] * (n - 1)), i32(range(1, n)), i32([text] * (n - 1)), begin=i32([whole] * (n - 1)), origin=origin)
    q, rows, at = draw(32, 4 * (n - 1), heads, width).cuda(), [0] + [4] * (n - 1), [0] + [text - whole] * (n - 1)
    cache.append(packed(k, [0] + [text] * (n - 1), rows), packed(v, [0] + [text] * (n - 1), rows), starts(rows), i32(at))
    got = cache.attend_shared(q, starts(rows), i32(at), cache, i32([1] + [n] * n), i32([text] + [0] * (n - 1)))
    full = stale(ad.Kv8Cache(n, heads, width, capacity=300, k_max=150))
    feed(full, k, v, [0] + [text] * (n - 1), 150)
    full.append(packed(k, [0] + [text] * (n - 1), rows), packed(v, [0] + [text] * (n - 1), rows), starts(rows), i32([0] + [text] * (n - 1)))
    want = full.attend(q, starts(rows), i32([0] + [text] * (n - 1)))
    for r in range(q.shape[0]):
        ref, size, dots = reference(f64(q[r]), [f64(t[0, :whole]) for t in (k, v)], [f64(t[1 + r // 4, whole:]) for t in (k, v)], text - whole + r % 4, "e4m3", width ** -0.5)
        tol = attend_tolerance(ref, size, dots, width)
        assert np.all(np.abs(f64(got[r]) - ref) <= tol) and np.all(np.abs(f64(want[r]) - ref) <= tol)


@pytest.mark.parametrize("fmt,q_heads", [("i8", 2), ("i8", 32), ("e4m3", 32)])     # (the latter: workgroups of 128 rows)
def test_scores_of_all_sizes_and_other_scales(fmt, q_heads):
    p = Problem(fmt, 64, 1, q_heads, [2], [300], [40, 60], [4, 4], True)
    p.q[1] = 0
    p.q[2] *= -40
    p.q[5] *= 30
    for scale in (None, -0.3, 0.0, 2.0):
        p.check(p.go(scale=scale), scale=scale)


@pytest.mark.parametrize("fmt,q_heads,capacity", [("e4m3", 1, None), ("e4m3", 1, 1100), ("e4m3", 32, None), ("i8", 32, None)])
def test_tokens_that_are_not_finite_spoil_what_sees_them_and_nothing_else(fmt, q_heads, capacity):
    clean = Problem(fmt, 64, 1, q_heads, [2, 2], [96, 64], [10, 40, 5, 50], [2, 2, 2, 2], True, capacity=capacity)
    want = clean.go()
    for where in ("text", "own"):
        p = Problem(fmt, 64, 1, q_heads, [2, 2], [96, 64], [10, 40, 5, 50], [2, 2, 2, 2], True, capacity=capacity)
        if where == "text":
            p.tv[0, 50, 0, 3] = INF
            feed(p.shared, p.tk, p.tv, p.text, 96)
        else:
            p.k[2, 6, 0, 3] = NAN                 # (the second row of sequence 2)
            p.cache.append(packed(p.k, p.lens, p.rows), packed(p.v, p.lens, p.rows), starts(p.rows), i32(p.lens))
        got = p.go()
        bad = [0, 1, 2, 3] if where == "text" else [5]
        for r in range(8):
            assert torch.isnan(got[r]).all() if r in bad else torch.equal(got[r], want[r]), (where, r)


@pytest.mark.parametrize("n_text,each", [(70, 2), (3, 50), (130, 1)])
def test_many_texts_with_and_without_bounds(n_text, each):
    rng = np.random.default_rng(n_text)
    text = [int(x) * 32 for x in rng.integers(0, 6, n_text)]
    counts = rng.integers(0, 2 * each + 1, n_text).tolist()
    counts[0] = max(counts[0], 1)
    n = sum(counts)
    lens, rows = rng.integers(0, 50, n).tolist(), rng.integers(0, 4, n).tolist()
    rows[0] = 2
    p = Problem("e4m3", 32, 2, 4, counts, text, lens, rows, False, capacity=6 * 32)
    got = p.go()
    p.check(got, every=7)
    together = max(sum(rows[a:b]) for a, b in zip(p.first, p.first[1:]))
    assert torch.equal(got, p.go(max_shared_rows=together, max_rows=3))


@pytest.mark.parametrize("group,capacity", FORMS)
def test_rows_lie_apart_and_what_is_no_row_stays(group, capacity):
    heads = 2 * group
    p = Problem("e4m3", 64, 2, heads, [2, 1], [64, 32], [30, 4, 64], [3, 0, 5], False, k_max=40, capacity=capacity)
    total, extra = 8, 2
    wide = torch.full((total + extra, 3, heads, 64), NAN, dtype=torch.bfloat16, device="cuda")
    wide[:total, 1] = p.q.cuda()
    out = torch.full((total + extra, 2, heads, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    got = p.go(q=wide[:, 1], out=out[:, 1], max_rows=5)
    p.check(got[:total])
    assert (out[total:] == 7).all() and (out[:, 0] == 7).all()
    # rows beyond the bound on a text's rows are left out, too
    out.fill_(7.0)
    p.go(q=wide[:, 1], out=out[:, 1], max_rows=5, max_shared_rows=4)
    assert torch.equal(out[:7, 1], got[:7]) and (out[7:, 1] == 7).all()


@pytest.mark.parametrize("group,capacity", FORMS)
def test_tables_are_held_to_the_buffers(group, capacity):
    """Tables that say something else than there is: no fault, and what they do not touch stays."""
    p = Problem("e4m3", 32, 1, group, [2, 2], [64, 32], [10, 20, 3, 40], [2, 2, 2, 2], False, k_max=8, capacity=capacity)
    want = p.go()
    for first, text in (([-5, 2, 9], [64, 32]), ([0, 2, 4], [10 ** 9, -7]), ([3, 1, 0], [64, 32]), ([4, 4, 4], [64, 32]), ([2 ** 31 - 1] * 3, [64, 32]), ([-2 ** 31] * 3, [64, 32])):
        p.go(seq_start=i32(first), shared_length=i32(text))
    out = torch.full_like(want, 7.0)
    p.go(row_start=i32([-4, -4, 0, 3, 100]), out=out, max_rows=8)
    p.go(row_start=i32([9, 8, 7, 6, 5]), max_rows=8)
    assert torch.equal(p.go(), want)


def test_shared_texts_are_refused():
    p = Problem("e4m3", 32, 2, 2, [2], [64], [10, 20], [2, 2], False)
    make = lambda **kw: ad.Kv8Cache(**dict(dict(n_seq=1, n_heads=2, head_width=32, capacity=64, k_max=4), **kw))  # noqa: E731
    for kw in (dict(shared=make(n_heads=1)), dict(shared=make(head_width=64)), dict(shared=make(format="i8")), dict(shared=None), dict(shared=make(n_seq=2)), dict(seq_start=i32([0])),
               dict(seq_start=i32([0, 2]).long()), dict(shared_length=i32([64]).cpu()), dict(shared_length=64), dict(q=p.q), dict(q=p.q.cuda().float()), dict(q=p.q.cuda()[:, :1]),
               dict(max_rows=-1), dict(max_rows=3, q=torch.cat([p.q.cuda()] * 2)), dict(max_shared_rows=-1), dict(max_keys=-1), dict(max_shared_keys=-1), dict(scale=NAN), dict(out=p.q.cuda()[:2])):
        with pytest.raises(ad.AdError) as e:
            p.go(**kw)
        assert e.value.code == ad.AD_EINVAL, kw
    closed = ad.Kv8Cache(2, 2, 32, 64, closed=True)
    with pytest.raises(ad.AdError, match="growing"):
        closed.attend_shared(p.q.cuda(), starts(p.rows), i32(p.lens), p.shared, i32([0, 2]), i32([64]))
    assert p.go(q=p.q.cuda()[:0], row_start=starts([0, 0])).shape == (0, 2, 32)


# ---- together --------------------------------------------------------------------------------------------------------------------------------
def step_inputs(seed, n, heads, width, vocab):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g).to(torch.bfloat16).cuda() for s in ((n, heads, width),) * 3] + [torch.rand(n, generator=g).cuda()]


def test_several_continuations_of_two_texts_drawn_together():
    """Texts taken in piece by piece, their last tokens copied to each continuation, then step by step: written, attended to, drawn; one continuation ends, and the last
    moves to its place.  Every attention and every token against the plain forms; the same captured and replayed."""
    heads, width, vocab, fmt = 2, 64, 700, "i8"
    text, each, steps = [75, 200], [3, 2], 6
    n = sum(each)
    tk, tv = draw(40, 2, 200, heads, width), draw(41, 2, 200, heads, width)
    out_w = draw(42, heads * width, vocab).float().cuda()
    owner = [g for g, m in enumerate(each) for _ in range(m)]
    whole = [t // 32 * 32 for t in text]
    shared = stale(ad.Kv8Cache(2, heads, width, capacity=200, k_max=64, format=fmt))
    feed(shared, tk, tv, text, 64)
    cache = stale(ad.Kv8Cache(n, heads, width, capacity=64, k_max=4, format=fmt))
    cache.copy(i32(owner), i32(range(n)), i32([text[g] for g in owner]), begin=i32([whole[g] for g in owner]), origin=shared)
    held = [[[f64(t[g, whole[g]:text[g]])] for t in (tk, tv)] for g in owner]
    lens, first = [text[g] - whole[g] for g in owner], [0, 3, 5]
    for step in range(steps):
        m = len(lens)
        live = [i for b in range(2) for i in range(first[b], first[b + 1])]
        rows = [1 if i in live else 0 for i in range(n)]
        q, k, v, u = step_inputs(50 + step, len(live), heads, width, vocab)
        at = i32(lens + [0] * (n - m))
        cache.append(k, v, starts(rows), at)
        o = cache.attend_shared(q, starts(rows), at, shared, i32(first), i32(text))
        logits = (o.float().view(len(live), -1) @ out_w) * 0.2
        temp, top_p = torch.full((len(live),), 0.8, device="cuda"), torch.full((len(live),), 0.9, device="cuda")
        tokens = ad.sample_tokens(logits, u, temperature=temp, top_p=top_p)
        for r, b in enumerate(live):
            g = 0 if b < first[1] else 1
            for j, t in enumerate((k, v)):
                held[b][j].append(f64(t[r:r + 1]))
            ref, size, dots = reference(f64(q[r]), [f64(t[g, :whole[g]]) for t in (tk, tv)], [np.concatenate(x) for x in held[b]], lens[b], fmt, width ** -0.5)
            assert np.all(np.abs(f64(o[r]) - ref) <= attend_tolerance(ref, size, dots, width)), (step, b)
            assert int(tokens[r]) == sample(f64(logits[r]), float(u[r]), float(np.float32(0.8)), 0, float(np.float32(0.9)))[0], (step, b)
        lens = [x + 1 for x in lens]
        if step == 2:                             # continuation 0 of the first text ends: its last one moves there
            cache.copy(i32([1, 2, 3, 4]), i32([0, 1, 2, 3]), i32(lens[1:]))
            lens, held, first = lens[1:], held[1:], [0, 2, 4]
    assert len(lens) == 4


def test_a_step_captured_and_replayed():
    """Append, attend over the shared text, draw, and a copy, in one graph; the tables change between the replays."""
    heads, width, n, steps, vocab = 2, 64, 4, 40, 300
    tk, tv = draw(60, 1, 96, heads, width), draw(61, 1, 96, heads, width)
    out_w = draw(62, heads * width, vocab).float().cuda()
    shared = stale(ad.Kv8Cache(1, heads, width, capacity=96, k_max=96))
    feed(shared, tk, tv, [96], 96)
    a, b = (stale(ad.Kv8Cache(n, heads, width, capacity=64, k_max=1)) for _ in range(2))
    q, k, v = (torch.zeros((n, heads, width), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    u, at, start, first, text = torch.zeros(n, device="cuda"), i32([0] * n), i32(range(n + 1)), i32([0, n]), i32([96])
    source, place, end = i32([0] * n), i32(range(n)), i32([0] * n)
    top_k = i32([20] * n)

    def step(cache, q, k, v, u, at, source, end):
        cache.append(k, v, start, at, max_rows=1)
        o = cache.attend_shared(q, start, at, shared, first, text, max_rows=1)
        tokens = ad.sample_tokens(o.float().view(n, -1) @ out_w, u, top_k=top_k)
        cache.copy(source, place, end)
        return o, tokens

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, q, k, v, u, at, source, end)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a, q, k, v, u, at, source, end)
    for i in range(steps):
        x = step_inputs(70 + i, n, heads, width, vocab)
        how = np.random.default_rng(i).integers(0, n, n)
        for to, t in zip((q, k, v, u), x):
            to.copy_(t)
        at.fill_(i)
        source.copy_(i32(how))
        end.fill_(i + 1)
        graph.replay()
        want = step(b, *x, i32([i] * n), i32(how), i32([i + 1] * n))
        assert all(torch.equal(g, w) for g, w in zip(got, want)), i
    for s in range(n):
        assert same(read(a, s, 0, steps), read(b, s, 0, steps))


def test_on_another_stream_and_dropped_while_it_waits():
    """Both caches of calls that wait on another stream keep their memory until these have run."""
    p = Problem("e4m3", 64, 2, 2, [3], [640], [10, 20, 30], [2, 2, 2], False)
    want = p.go()
    moved = torch.cat([read(p.cache, b, 0, 12) for b in (0, 1)])
    target = ad.Kv8Cache(2, 2, 64, capacity=64, k_max=4)
    args = p.q.cuda(), starts(p.rows), i32(p.lens), i32(p.first), i32(p.text), i32([0, 1]), i32([0, 1]), i32([12, 12])
    side, busy = torch.cuda.Stream(), torch.zeros(4096, 4096, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    cache, shared = p.cache, p.shared
    del p
    with torch.cuda.stream(side):
        for _ in range(40):
            busy = busy @ busy
        got = cache.attend_shared(args[0], args[1], args[2], shared, args[3], args[4])
        target.copy(args[5], args[6], args[7], origin=cache)
    sizes = cache.memory.numel(), shared.memory.numel()
    del cache, shared
    others = [torch.full((size,), 0x55, dtype=torch.uint8, device="cuda") for size in sizes for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 8
    assert same(torch.cat([read(target, b, 0, 12) for b in (0, 1)]), moved)
