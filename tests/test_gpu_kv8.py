"""Key/value caches in 8 bits through the public entry points, against the plain 64-bit form."""
import numpy as np
import pytest

import paper_2205_10350_amd as ad
from kv8_reference import BLOCK, attend, attend_tolerance, tokens_as_read

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
    return t.double().numpy()


def packed(t, at, n):
    """Rows at[b] .. at[b] + n[b] - 1 of t [batch, tokens, ..], on the GPU."""
    return torch.cat([t[b, a:a + m] for b, (a, m) in enumerate(zip(at, n))]).cuda()


def stale(cache):
    """Whatever lies in the memory must not matter: NaN patterns of every type."""
    cache.memory.fill_(0xFF)
    return cache


def feed(cache, k, v, lens, step):
    """Tokens [0, lens[b]) of k, v, at most `step` of a sequence in a call."""
    for at in range(0, max(lens), step):
        part = [max(0, min(n - at, step)) for n in lens]
        begin = [min(at, n) for n in lens]
        cache.append(packed(k, begin, part), packed(v, begin, part), starts(part), i32(begin))


def read_all(cache, lens, dtype=torch.float32):
    k, v = cache.read(starts(lens), i32([0] * len(lens)), i32(lens), rows=sum(lens), dtype=dtype)
    return k, v


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("width,heads", [(32, 3), (64, 2), (128, 1)])
@pytest.mark.parametrize("step", [1, 7, 33])
def test_written_values_read_back(fmt, width, heads, step):
    lens = [70, 0, 1, 31, 32, 33, 64]
    k, v = draw(1, len(lens), 70, heads, width), draw(2, len(lens), 70, heads, width, spread=1.0)
    cache = stale(ad.Kv8Cache(len(lens), heads, width, capacity=70, k_max=step, format=fmt))
    feed(cache, k, v, lens, step)
    for dtype in (torch.float32, torch.bfloat16):
        # (an incomplete block's tokens: as the next row reads them)
        whole = cache.read(starts(lens), i32([0] * len(lens)), i32(lens), rows=sum(lens), dtype=dtype)
        at = 0
        for b, n in enumerate(lens):
            for got, t in zip(whole, (k, v)):
                want = torch.tensor(tokens_as_read(f64(t[b, :n]), n, fmt))
                # (a value is byte * scale, one rounding in fp32; as float64 products of a byte and an fp32 scale, rounded once, that is the same)
                assert torch.equal(got[at:at + n].cpu(), want.to(torch.float32).to(dtype)), (b, n)
            at += n


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
def test_written_values_at_the_edges_of_the_types(fmt):
    """Blocks of zeros, of the smallest and largest bf16 numbers, with halves between two steps."""
    w = 32
    blocks = []
    for most in (0.0, 1.0, 448.0, 449.0, 2.0 ** -126, 2.0 ** -133, 3.3895313892515355e38, 127.0, 3.0):
        x = np.zeros((BLOCK, w))
        x[0, 0] = most
        x[1:17, :] = most * np.arange(16 * w).reshape(16, w) / 512.0      # halves and everything between
        x[17:, 1:] = -most * np.random.default_rng(5).random((15, w - 1))
        blocks.append(torch.tensor(x, dtype=torch.float64).to(torch.float32).to(torch.bfloat16))
    t = torch.cat(blocks)[None, :, None, :].contiguous()
    n = t.shape[1]
    cache = stale(ad.Kv8Cache(1, 1, w, capacity=n, k_max=n, format=fmt))
    feed(cache, t, t, [n], n)
    want = tokens_as_read(f64(t[0]), n, fmt)
    for got in read_all(cache, [n]):
        got = got.cpu().double().numpy()
        # (scales below the normal numbers are themselves rounded: half a step of the smallest subnormal, 127 times)
        assert np.allclose(got, want.astype(np.float32), rtol=0, atol=128 * 2.0 ** -150), np.abs(got - want).max()


@pytest.mark.parametrize("closed", [False, True])
def test_a_token_that_is_not_finite_spoils_what_reads_it_and_nothing_else(closed):
    n, w, bad = 80, 64, 40
    k, v, q = draw(3, 1, n, 1, w), draw(4, 1, n, 1, w), draw(5, 1, n, 1, w)
    for which, value in ((0, NAN), (1, NAN), (0, INF), (1, -INF)):
        kk, vv = k.clone(), v.clone()
        (kk, vv)[which][0, bad, 0, 5] = value
        out = {}
        for name, (a, b) in {"clean": (k, v), "bad": (kk, vv)}.items():
            cache = stale(ad.Kv8Cache(1, 1, w, capacity=n, k_max=n, closed=closed))
            feed(cache, a, b, [n], n)
            out[name] = cache.attend(q[0].cuda(), starts([n]), i32([n if closed else 0])).cpu()
        assert torch.isfinite(out["clean"]).all()
        sees = np.ones(n, bool) if closed else np.arange(n) >= bad
        assert torch.isnan(out["bad"][sees]).all()
        assert torch.equal(out["bad"][~sees], out["clean"][~sees])


def test_rejected_tokens_leave_nothing_behind():
    """Blocks of drafted tokens, some NaN, taken back after each call: values and attention are those of the kept tokens alone, bit for bit."""
    rng = np.random.default_rng(7)
    n, w, heads = 150, 64, 2
    k, v, q = draw(8, 1, n, heads, w), draw(9, 1, n, heads, w), draw(10, 1, n, heads, w)
    plain = stale(ad.Kv8Cache(1, heads, w, capacity=n + 40, k_max=40, format="i8"))
    feed(plain, k, v, [n], 1)
    cache = stale(ad.Kv8Cache(1, heads, w, capacity=n + 40, k_max=40, format="i8"))
    at, outs = 0, []
    while at < n:
        rows, keep = int(rng.integers(1, 41)), int(rng.integers(1, 12))
        keep = min(keep, rows, n - at)
        kk, vv, qq = (torch.cat((t[0, at:at + keep], draw(int(rng.integers(1 << 20)), rows - keep, heads, w) * 50)) for t in (k, v, q))
        if rows > keep:
            kk[keep] = NAN
            vv[-1] = INF
        cache.append(kk.cuda(), vv.cuda(), starts([rows]), i32([at]))
        outs.append(cache.attend(qq.cuda(), starts([rows]), i32([at]))[:keep])
        at += keep
    for a, b in zip(read_all(cache, [n]), read_all(plain, [n])):
        assert torch.equal(a, b)
    alone = torch.cat([plain_row(k, v, q, i, heads, w, n) for i in range(n)])
    assert torch.equal(torch.cat(outs), alone)


def plain_row(k, v, q, i, heads, w, n, fmt="i8"):
    cache = ad.Kv8Cache(1, heads, w, capacity=n + 40, k_max=40, format=fmt)
    feed(cache, k, v, [i + 1], 40)
    return cache.attend(q[0, i:i + 1].cuda(), starts([1]), i32([i]))


CASES = [
    # format, width, heads, query heads, lengths before the block, rows of the block
    ("e4m3", 64, 2, 2, [0, 1, 31, 32, 33, 100], [1, 1, 1, 1, 1, 1]),
    ("i8", 64, 2, 2, [0, 5, 30, 63, 255, 256], [25, 3, 0, 40, 7, 1]),
    ("e4m3", 32, 3, 6, [511, 0, 700], [9, 70, 33]),
    ("i8", 32, 1, 1, [1030], [64]),
    ("e4m3", 128, 1, 4, [1025, 3, 256], [1, 2, 5]),
    ("i8", 128, 2, 10, [40, 600], [25, 3]),
    ("e4m3", 64, 1, 16, [2100], [3]),
]


def check(got, q, k, v, at, rows, fmt, closed=False):
    got = got.float().cpu().numpy().astype(np.float64)
    r = 0
    for b, (n, m) in enumerate(zip(at, rows)):
        for i in range(m):
            kk, vv = f64(k[b]), f64(v[b])
            if closed:
                kk, vv = kk[:n], vv[:n]
            ref, size, dots = attend(f64(q[r]), kk, vv, n + i, fmt, q.shape[2] ** -0.5, closed)
            tol = attend_tolerance(ref, size, dots, q.shape[2])
            assert np.all(np.abs(got[r] - ref) <= tol), (b, i, np.max(np.abs(got[r] - ref) / tol))
            r += 1


@pytest.mark.parametrize("fmt,width,heads,q_heads,at,rows", CASES)
def test_attention_of_a_growing_cache(fmt, width, heads, q_heads, at, rows):
    most = max(a + m for a, m in zip(at, rows))
    k, v, q = draw(11, len(at), most, heads, width), draw(12, len(at), most, heads, width), draw(13, sum(rows), q_heads, width)
    cache = stale(ad.Kv8Cache(len(at), heads, width, capacity=most + 5, k_max=max(rows + [1]), format=fmt))
    feed(cache, k, v, at, max(rows + [1]))
    cache.append(packed(k, at, rows), packed(v, at, rows), starts(rows), i32(at))
    got = cache.attend(q.cuda(), starts(rows), i32(at))
    check(got, q, k, v, at, rows, fmt)
    # the same bits whatever the bounds of the launch, token by token, and alone
    assert torch.equal(got, cache.attend(q.cuda(), starts(rows), i32(at), max_rows=max(rows), max_keys=most))
    r = 0
    for b, (n, m) in enumerate(zip(at, rows)):
        for i in range(m):
            if i in (0, m // 2, m - 1):
                other = [0] * len(at)
                other[b] = 1
                one = cache.attend(q[r + i:r + i + 1].cuda(), starts(other), i32([n + i] * len(at)))
                assert torch.equal(one, got[r + i:r + i + 1]), (b, i)
        r += m


@pytest.mark.parametrize("fmt,width,heads,q_heads,at,rows", CASES)
def test_attention_of_a_closed_cache(fmt, width, heads, q_heads, at, rows):
    most = max(at)
    k, v, q = draw(14, len(at), most, heads, width), draw(15, len(at), most, heads, width), draw(16, sum(rows), q_heads, width)
    cache = stale(ad.Kv8Cache(len(at), heads, width, capacity=most, format=fmt, closed=True))
    feed(cache, k, v, at, most)
    got = cache.attend(q.cuda(), starts(rows), i32(at))
    check(got, q, k, v, at, rows, fmt, closed=True)
    for n, lo, m in zip(at, np.cumsum([0] + rows), rows):
        if n == 0:
            assert (got[lo:lo + m] == 0).all()
    assert torch.equal(got, cache.attend(q.cuda(), starts(rows), i32(at), max_rows=max(rows), max_keys=most))


def test_scores_of_all_sizes():
    """Scores of +-300 and of nothing: the running maximum moves, and most keys weigh nothing."""
    n, w = 300, 64
    k, v, q = draw(17, 1, n, 1, w), draw(18, 1, n, 1, w), draw(19, 4, 1, w) * 12
    q[1] = 0
    q[2] *= -8
    cache = stale(ad.Kv8Cache(1, 1, w, capacity=n, k_max=n))
    feed(cache, k, v, [n], n)
    got = cache.attend(q.cuda(), starts([4]), i32([n - 4]))
    check(got, q, k, v, [n - 4], [4], "e4m3")


def test_rows_lie_apart_and_what_is_no_row_stays():
    """Keys, values and queries out of one fused [rows, 3 d] tensor; outputs into a wider one; rows behind the last sequence."""
    heads, w, rows, at = 2, 64, [3, 0, 5], [30, 4, 64]
    most, total, extra = 80, 8, 2
    k, v = draw(20, 3, most, heads, w), draw(21, 3, most, heads, w)
    q = draw(22, total, heads, w)
    cache = stale(ad.Kv8Cache(3, heads, w, capacity=most, k_max=40))
    feed(cache, k, v, at, 40)
    fused = torch.full((total + extra, 3, heads, w), NAN, dtype=torch.bfloat16, device="cuda")
    fused[:total, 0], fused[:total, 1], fused[:total, 2] = q.cuda(), packed(k, at, rows), packed(v, at, rows)
    wide = torch.full((total + extra, 2, heads, w), 7.0, dtype=torch.bfloat16, device="cuda")
    cache.append(fused[:, 1], fused[:, 2], starts(rows), i32(at), max_rows=5)
    got = cache.attend(fused[:, 0], starts(rows), i32(at), max_rows=5, out=wide[:, 1])
    check(got[:total], q, k, v, at, rows, "e4m3")
    assert (wide[total:] == 7).all() and (wide[:, 0] == 7).all()
    kr, vr = cache.read(starts(rows), i32(at), i32([a + m for a, m in zip(at, rows)]), rows=total + extra)
    assert torch.isfinite(kr[:total]).all() and torch.isfinite(vr[:total]).all()


def test_tables_are_held_to_the_buffers():
    """Lengths and starts that say more than there is: what does not fit is left out, and the rest is right."""
    heads, w, cap = 1, 32, 40
    k, v, q = draw(23, 2, cap, heads, w), draw(24, 2, cap, heads, w), draw(25, 8, heads, w)
    cache = stale(ad.Kv8Cache(2, heads, w, capacity=cap, k_max=cap))
    feed(cache, k, v, [cap, 20], cap)
    before = cache.memory.clone()
    rows = draw(26, 8, heads, w).cuda()
    for start, at in (([0, -3, 4], [3, -1]), ([9, 12, 20], [0, 0]), ([0, 4, 8], [cap, cap + 9]), ([5, 2, 1], [0, 0])):
        cache.append(rows, rows, i32(start), i32(at), max_rows=8)
        assert torch.equal(cache.memory, before), start
    out = torch.full((8, heads, w), 7.0, dtype=torch.bfloat16, device="cuda")
    cache.attend(q.cuda(), i32([-4, 0, 100]), i32([3, 12]), out=out, max_rows=8)
    check(out, q, k[1:], v[1:], [12], [8], "e4m3")


def test_captured_and_replayed():
    heads, w, n = 2, 64, 90
    k, v, q = draw(27, 2, n, heads, w), draw(28, 2, n, heads, w), draw(29, 2, n, heads, w)
    eager = ad.Kv8Cache(2, heads, w, capacity=n, k_max=3)
    cache = stale(ad.Kv8Cache(2, heads, w, capacity=n, k_max=3))
    kk, vv, qq = (torch.zeros((6, heads, w), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    start, at = i32([0, 3, 6]), i32([0, 0])
    out = torch.zeros_like(qq)
    ws_free = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(kk, vv, start, at, max_rows=3)
        cache.attend(qq, start, at, max_rows=3, out=out)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(ws_free):
        cache.append(kk, vv, start, at, max_rows=3)
        cache.attend(qq, start, at, max_rows=3, out=out)
    for i in range(0, n, 3):
        rows = [packed(t, [i, i], [3, 3]) for t in (k, v, q)]
        for to, x in zip((kk, vv, qq), rows):
            to.copy_(x)
        at.fill_(i)
        ws_free.replay()
        eager.append(rows[0], rows[1], start, i32([i, i]), max_rows=3)
        assert torch.equal(out, eager.attend(rows[2], start, i32([i, i]), max_rows=3)), i


@pytest.mark.parametrize("closed", [False, True])
@pytest.mark.parametrize("n_seq,heads,q_heads", [(40, 1, 1), (150, 2, 6)])
def test_many_sequences_with_and_without_a_bound(n_seq, heads, q_heads, closed):
    """Blocks, tiles and rows looked up in the table (no bound: mostly ones that are not there) and by sequence, splits and empty sequences among them."""
    w, cap = 32, 1400
    rng = np.random.default_rng(n_seq)
    lens = [0] + [int(x) for x in rng.integers(1, 90, n_seq - 2)] + [1200]
    lens[7] = 0
    k, v = draw(40, n_seq, cap, heads, w), draw(41, n_seq, cap, heads, w)
    wide, tight = (ad.Kv8Cache(n_seq, heads, w, capacity=cap, k_max=cap, closed=closed) for _ in range(2))
    at = i32([0] * n_seq)
    kk, vv = packed(k, [0] * n_seq, lens), packed(v, [0] * n_seq, lens)
    wide.append(kk, vv, starts(lens), at)
    for b in range(n_seq):                                                # one sequence a call
        one = [lens[b] if i == b else 0 for i in range(n_seq)]
        lo = sum(lens[:b])
        if lens[b]:
            tight.append(kk[lo:lo + lens[b]], vv[lo:lo + lens[b]], starts(one), at, max_rows=lens[b])
    for got, want in zip(read_all(wide, lens), read_all(tight, lens)):
        assert torch.equal(got, want)
    some = wide.read(starts(lens), at, i32(lens), rows=sum(lens), max_rows=max(lens), dtype=torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(some, read_all(wide, lens)))
    rows = [min(n, int(x)) for n, x in zip(lens, rng.integers(0, 40, n_seq))]
    before = lens if closed else [n - r for n, r in zip(lens, rows)]
    q = draw(42, sum(rows), q_heads, w).cuda()
    got = wide.attend(q, starts(rows), i32(before))
    assert torch.equal(got, tight.attend(q, starts(rows), i32(before), max_rows=max(rows)))
    lo = 0
    for b in range(n_seq):                                                # and each sequence by itself
        if rows[b] and b % 9 == 0 or b == n_seq - 1:
            one = [rows[b] if i == b else 0 for i in range(n_seq)]
            assert torch.equal(got[lo:lo + rows[b]], tight.attend(q[lo:lo + rows[b]].contiguous(), starts(one), i32(before), max_rows=max(rows[b], 1)) if rows[b] else got[lo:lo])
        lo += rows[b]


def test_on_another_stream():
    heads, w, n = 2, 64, 400
    k, v, q = draw(30, 1, n, heads, w), draw(31, 1, n, heads, w), draw(32, 5, heads, w).cuda()
    want = ad.Kv8Cache(1, heads, w, capacity=n, k_max=n)
    feed(want, k, v, [n], n)
    side = torch.cuda.Stream()
    kk, vv, start, at = packed(k, [0], [n]), packed(v, [0], [n]), starts([n]), i32([0])
    some, tail = starts([5]), i32([n - 5])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache = ad.Kv8Cache(1, heads, w, capacity=n, k_max=n)
        cache.append(kk, vv, start, at)
        got = cache.attend(q, some, tail)
    side.synchronize()
    assert torch.equal(got, want.attend(q, some, tail))


def test_memory_outlives_the_calls_of_another_stream():
    """A cache that is dropped while another stream's calls on it wait keeps its memory until they have run."""
    heads, w, n = 2, 64, 4000
    k, v, q = draw(33, 1, n, heads, w), draw(34, 1, n, heads, w), draw(35, 5, heads, w).cuda()
    cache = ad.Kv8Cache(1, heads, w, capacity=n, k_max=n)
    feed(cache, k, v, [n], n)
    some, tail = starts([5]), i32([n - 5])
    want = cache.attend(q, some, tail)
    side, busy = torch.cuda.Stream(), torch.zeros(4096, 4096, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(40):
            busy = busy @ busy
        got = cache.attend(q, some, tail)
    size = cache.memory.numel()
    del cache
    others = [torch.full((size,), 0x55, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(others) == 4


def test_a_long_cache_past_32_bits():
    """Offsets of the last sequence lie beyond 4 GiB."""
    heads, w, cap, n_seq = 8, 128, 1 << 17, 17
    cache = ad.Kv8Cache(n_seq, heads, w, capacity=cap, k_max=64)
    assert cache.memory.numel() > 1 << 32
    k, v, q = draw(33, 1, 70, heads, w), draw(34, 1, 70, heads, w), draw(35, 4, heads, w)
    base = cap - 96
    for lo, m in ((0, 64), (64, 6)):
        rows = [0] * (n_seq - 1) + [m]
        cache.append(k[0, lo:lo + m].cuda(), v[0, lo:lo + m].cuda(), starts(rows), i32([0] * (n_seq - 1) + [base + lo]))
    got = cache.read(starts([0] * (n_seq - 1) + [70]), i32([0] * (n_seq - 1) + [base]), i32([0] * (n_seq - 1) + [base + 70]), rows=70, dtype=torch.float32)
    for g, t in zip(got, (k, v)):
        assert torch.equal(g.cpu(), torch.tensor(tokens_as_read(f64(t[0]), 70, "e4m3")).to(torch.float32))


def test_rows_that_no_sequence_may_have_are_refused_by_default():
    """Without max_rows: more packed rows than the sequences may have in a call, of which some would be dropped."""
    heads, w = 2, 64
    k, v, q = (draw(54 + i, 100, heads, w).cuda() for i in range(3))
    one = ad.Kv8Cache(1, heads, w, capacity=128)                       # (k_max = 1)
    two = ad.Kv8Cache(2, heads, w, capacity=128, k_max=25)
    for cache, rows in ((one, [100]), (one, [2]), (two, [25, 26])):
        n = sum(rows)
        at = i32([0] * len(rows))
        with pytest.raises(ad.AdError, match="max_rows") as e:
            cache.append(k[:n], v[:n], starts(rows), at)
        assert e.value.code == ad.AD_EINVAL
        with pytest.raises(ad.AdError, match="max_rows"):
            cache.attend(q[:n], starts(rows), at)
    # as many as there may be; rows behind the last sequence, where the caller says how many a sequence has
    two.append(k[:50], v[:50], starts([25, 25]), i32([0, 0]))
    one.append(k, v, starts([1]), i32([0]), max_rows=1)
    assert torch.equal(one.read(starts([1]), i32([0]), i32([1]), rows=1)[0][0], k[0])
    closed = ad.Kv8Cache(1, heads, w, capacity=128, closed=True)
    with pytest.raises(ad.AdError, match="max_rows"):
        closed.append(draw(57, 129, heads, w).cuda(), draw(58, 129, heads, w).cuda(), starts([129]), i32([0]))
    closed.append(k, v, starts([100]), i32([0]))
    many = closed.attend(torch.cat([q] * 3), starts([300]), i32([100]))    # (queries over a memory: as many as one likes)
    assert torch.equal(many[:100], many[200:])


def test_a_bound_above_the_rows_is_a_bound():
    """max_rows as a program sets it once, for its longest blocks, in a call of few rows."""
    heads, w = 2, 64
    k, v, q = (draw(60 + i, 3, heads, w).cuda() for i in range(3))
    got = []
    for most in (3, 25):
        cache = stale(ad.Kv8Cache(1, heads, w, capacity=40, k_max=25))
        cache.append(k, v, starts([3]), i32([0]), max_rows=most)
        got.append((cache.attend(q, starts([3]), i32([0]), max_rows=most), *cache.read(starts([3]), i32([0]), i32([3]), rows=3, max_rows=most)))
        assert cache.attend(q[:0], starts([0]), i32([3]), max_rows=most).shape == (0, heads, w)
        with pytest.raises(ad.AdError):
            cache.append(k, v, starts([3]), i32([0]), max_rows=-1)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def check_scaled(got, q, k, v, at, rows, fmt, scale, closed):
    got = got.float().cpu().numpy().astype(np.float64)
    r = 0
    for b, (n, m) in enumerate(zip(at, rows)):
        for i in range(m):
            kk, vv = f64(k[b]), f64(v[b])
            if closed:
                kk, vv = kk[:n], vv[:n]
            ref, size, dots = attend(f64(q[r]), kk, vv, n + i, fmt, scale, closed)
            tol = attend_tolerance(ref, size, dots, q.shape[2])
            assert np.all(np.abs(got[r] - ref) <= tol), (b, i, np.max(np.abs(got[r] - ref) / tol))
            r += 1


@pytest.mark.parametrize("scale", [-0.2, 0.0, 0.7])
@pytest.mark.parametrize("closed", [False, True])
@pytest.mark.parametrize("fmt,width,heads,q_heads,at,rows", CASES[:5])
def test_attention_with_a_scale_of_any_sign(fmt, width, heads, q_heads, at, rows, closed, scale):
    """A negative scale prefers the smallest products, 0 weighs every visible key alike; tiles over a block's border, where some rows see a block and some do not."""
    most = max(a + m for a, m in zip(at, rows))
    k, v, q = draw(51, len(at), most, heads, width), draw(52, len(at), most, heads, width), draw(53, sum(rows), q_heads, width)
    cache = stale(ad.Kv8Cache(len(at), heads, width, capacity=most, k_max=max(rows + [1]), format=fmt, closed=closed))
    if closed:
        feed(cache, k, v, at, max(at))
    else:
        feed(cache, k, v, at, max(rows + [1]))
        cache.append(packed(k, at, rows), packed(v, at, rows), starts(rows), i32(at))
    check_scaled(cache.attend(q.cuda(), starts(rows), i32(at), scale=scale), q, k, v, at, rows, fmt, scale, closed)
