"""Tables that say something else than there is: nothing beside the rows that a valid sequence owns is written, and those are right.  Outputs lie within larger buffers.
And tables that change between the replays of a captured step."""
import numpy as np
import pytest

import paper_2205_10350_amd as ad
from kv8_reference import attend_tolerance
from test_gpu_kv8_shared import FORMS, Problem, draw, f64, feed, i32, read, reference, same, stale, starts
from truncate_reference import kept, sample

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

GUARD = 5


def guarded(rows, *shape, dtype=torch.bfloat16):
    """(whole buffer filled with 7, its middle `rows` rows)"""
    whole = torch.full((rows + 2 * GUARD, *shape), 7, dtype=dtype, device="cuda")
    return whole, whole[GUARD:GUARD + rows]


def untouched(whole):
    return (whole[:GUARD] == 7).all() and (whole[-GUARD:] == 7).all()


LEAST, MOST = -2 ** 31, 2 ** 31 - 1
# row_start of four sequences over 8 packed rows, differences of which leave 32 bits; the rows that they give a sequence, if any
ENDS = [([LEAST, LEAST + 5, LEAST + 9, LEAST + 9, LEAST + 10], ()), ([LEAST, 0, LEAST, 0, LEAST], ()), ([8, LEAST + 108, 8, LEAST + 1000, 8], ()), ([MOST, LEAST, MOST, LEAST, MOST], ()),
        ([-1, MOST, LEAST, -8, LEAST + 8], ()), ([LEAST] * 4 + [MOST], ()), ([0, 2, 2, LEAST, LEAST + 8], (0, 1))]


@pytest.mark.parametrize("start,owned", ENDS)
def test_row_tables_at_the_ends_of_32_bits(start, owned):
    """Appended, read, attended to (query heads that share a head among them, whose number the rows are multiplied by), over a growing cache, a closed one and shared texts."""
    heads, width = 1, 32
    k, v = draw(90, 8, heads, width).cuda(), draw(91, 8, heads, width).cuda()
    mine = torch.zeros(8, dtype=torch.bool, device="cuda")
    mine[list(owned)] = True
    for closed in (False, True):
        cache = stale(ad.Kv8Cache(4, heads, width, capacity=64, k_max=8, closed=closed))
        cache.append(k, v, starts([2, 2, 2, 2]), i32([0] * 4))
        before = cache.memory.clone()
        if not owned:
            cache.append(k, v, i32(start), i32([0 if closed else 2] * 4), max_rows=8)
            assert torch.equal(cache.memory, before)
        cache.read(i32(start), i32([0] * 4), i32([2] * 4), rows=8)
        for group in (1, 2, 4, 32):
            q = draw(92, 8, heads * group, width).cuda()
            whole, out = guarded(8, heads * group, width)
            cache.attend(q, i32(start), i32([2 if closed else 0] * 4), max_rows=8, out=out)
            assert untouched(whole) and (out[~mine] == 7).all() and torch.isfinite(out).all(), (closed, group)
    for group, capacity in FORMS:
        for each in (group, 4 * group):
            p = Problem("e4m3", width, heads, each, [2, 2], [64, 32], [10, 20, 3, 40], [2, 2, 2, 2], False, k_max=8, capacity=capacity)
            whole, out = guarded(8, each, width)
            p.go(row_start=i32(start), out=out, max_rows=8)
            assert untouched(whole) and (out[~mine] == 7).all(), (each, capacity)
            if owned:
                assert torch.equal(out[mine], p.go(row_start=i32([0, 2, 2, 2, 2]), max_rows=8)[mine])


@pytest.mark.parametrize("group,capacity", FORMS)
def test_attention_writes_the_rows_of_valid_sequences_alone(group, capacity):
    p = Problem("e4m3", 32, 1, group, [2, 2], [64, 32], [10, 20, 3, 40], [2, 2, 2, 2], False, k_max=8, capacity=capacity)
    right = p.go()
    # texts' tables: those that mean the right ones, none, and others
    for first, text, like in (([-5, 2, 9], [64, 32], dict()), ([0, 2, 4], [10 ** 9, -7], dict(shared_length=i32([p.shared.cfg.capacity, 0]))), ([4, 4, 4], [64, 32], dict(shared_length=i32([0, 0]))),
                              ([2 ** 31 - 1] * 3, [64, 32], dict(shared_length=i32([0, 0]))), ([3, 1, 0], [64, 32], None), ([-2 ** 31] * 3, [64, 32], None)):
        whole, out = guarded(8, group, 32)
        p.go(seq_start=i32(first), shared_length=i32(text), out=out)
        assert untouched(whole), first
        if like is not None and not (text[0] > 64 and p.shared.cfg.capacity > 64):     # (tokens that were never written are not compared)
            assert torch.equal(out, p.go(**like)), first
    # rows' tables
    for start, like, owned in (([-4, -4, 0, 3, 100], [0, 0, 0, 3, 8], range(8)), ([9, 8, 7, 6, 5], None, ()), ([100, 100, 100, 100, 200], None, ()), ([-9, -7, -5, -3, -1], None, ()),
                               ([0, 2, 2, 2, 5], [0, 2, 2, 2, 5], range(5))):
        whole, out = guarded(8, group, 32)
        p.go(row_start=i32(start), out=out, max_rows=8)
        assert untouched(whole), start
        mine = torch.zeros(8, dtype=torch.bool, device="cuda")
        mine[list(owned)] = True
        assert (out[~mine] == 7).all(), start
        if like is not None:
            # (rows behind those that were appended see memory that was never written: the same bits, NaN among them)
            assert torch.equal(out[mine].view(torch.int16), p.go(row_start=i32(like), max_rows=8)[mine].view(torch.int16)), start
    assert torch.equal(p.go(), right)


@pytest.mark.parametrize("vocab", [600, 5000])
@pytest.mark.parametrize("n_seq", [3, 70])
def test_truncation_writes_the_rows_of_valid_sequences_alone(n_seq, vocab):
    rng = np.random.default_rng(n_seq)
    n = 40
    x = torch.tensor(rng.standard_normal((n, vocab)) * 3, dtype=torch.float32).cuda()
    u = torch.tensor(rng.random(n), dtype=torch.float32).cuda()
    k = i32(np.arange(n_seq) % 7 + 1)
    xs = f64(x)
    tables = [([-5] * n_seq + [-2], {}), ([n] * (n_seq + 1), {}), (list(range(n_seq, -1, -1)), {}), ([0] * n_seq + [n + 100], {r: n_seq - 1 for r in range(n)}),
              ([-2 ** 31] + [3] * n_seq, {r: 0 for r in range(3)}), ([2] * n_seq + [2 ** 31 - 1], {r: n_seq - 1 for r in range(2, n)}), ([5, 9] + [9] * (n_seq - 1), {r: 0 for r in range(5, 9)})]
    for start, owner in tables:
        start = i32(start)
        whole, out = guarded(n, vocab, dtype=torch.float32)
        ad.truncate_scores(x, top_k=k, row_start=start, out=out)
        (all_t, tokens), (all_p, probs) = guarded(n, dtype=torch.int32), guarded(n, dtype=torch.float32)
        stream = torch.cuda.current_stream().cuda_stream
        assert ad.lib().ad_sample_tokens(x.data_ptr(), ad.AD_F32, vocab, vocab, None, k.data_ptr(), None, None, start.data_ptr(), n_seq, u.data_ptr(), n, tokens.data_ptr(), probs.data_ptr(),
                                         stream) == ad.AD_OK
        assert untouched(whole) and untouched(all_t) and untouched(all_p), start
        for r in range(n):
            if r not in owner:
                assert (out[r] == 7).all() and tokens[r] == 7 and probs[r] == 7, (start, r)
                continue
            of = 1.0, int(k[owner[r]]), 1.0, 0.0
            assert int(tokens[r]) == sample(xs[r], float(u[r]), *of)[0], (start, r)
            assert np.array_equal(f64(out[r]), np.where(kept(xs[r], *of), xs[r], -np.inf)), (start, r)


@pytest.mark.parametrize("group,capacity", FORMS)
def test_a_step_of_two_texts_replayed_with_other_tables(group, capacity):
    """Append, attend, draw and move together in one graph: which text a continuation has, how long the texts are, which continuations have a row and which sequences move change between the
    replays.  Attention and tokens against the plain forms, caches against a twin that is worked on eagerly."""
    heads, width, n, vocab, fmt = 1, 64, 5, 300, "e4m3"
    tk, tv = draw(80, 2, 192, heads, width), draw(81, 2, 192, heads, width)
    q_heads = heads * group
    out_w = draw(82, q_heads * width, vocab).float().cuda()
    shared = stale(ad.Kv8Cache(2, heads, width, capacity=capacity or 192, k_max=192, format=fmt))
    feed(shared, tk, tv, [192, 160], 192)
    a, b = (stale(ad.Kv8Cache(n, heads, width, capacity=64, k_max=1, format=fmt)) for _ in range(2))
    zeros = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    q, k, v, u = zeros(n, q_heads, width), zeros(n, heads, width), zeros(n, heads, width), zeros(n, dtype=torch.float32)
    tables = [zeros(m, dtype=torch.int32) for m in (n + 1, n, 3, 2, n, n, n)]
    top_k = i32([20] * n)

    def step(cache, q, k, v, u, start, at, first, text, source, place, end):
        cache.append(k, v, start, at, max_rows=1)
        o = cache.attend_shared(q, start, at, shared, first, text, max_rows=1)
        logits = o.float().view(n, -1) @ out_w * 0.2
        tokens = ad.sample_tokens(logits, u, top_k=top_k)
        cache.copy(source, place, end)
        return o, logits, tokens

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, q, k, v, u, *tables)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a, q, k, v, u, *tables)
    a.memory.fill_(0xFF)
    lens, held = [0] * n, [[[], []] for _ in range(n)]
    rng = np.random.default_rng(83)
    for i in range(36):
        split = sorted(rng.integers(0, n + 1, 3).tolist())
        text = [int(rng.integers(0, 7)) * 32, int(rng.integers(0, 6)) * 32]
        rows = (rng.random(n) < 0.8).astype(int).tolist()
        rows = [r if m < 64 else 0 for r, m in zip(rows, lens)]
        total = sum(rows)
        x = [t.cuda() for t in (draw(100 + 4 * i, n, q_heads, width), draw(101 + 4 * i, n, heads, width), draw(102 + 4 * i, n, heads, width))] + [torch.tensor(rng.random(n), dtype=torch.float32).cuda()]
        after = [m + r for m, r in zip(lens, rows)]
        how = rng.integers(0, n, n) if i % 3 == 2 else np.arange(n)
        now = [starts(rows), i32(lens), i32(split), i32(text), i32(how), i32(range(n)), i32([after[j] for j in how])]
        for to, t in zip([q, k, v, u] + tables, x + now):
            to.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        step(b, *x, *now)
        r = 0
        for s in range(n):
            if not rows[s]:
                continue
            g = next((g for g in range(2) if split[g] <= s < split[g + 1]), None)
            for j, t in enumerate(x[1:3]):
                held[s][j].append(f64(t[r:r + 1]))
            front = [f64(t[g, :text[g]]) if g is not None else f64(t[0, :0]) for t in (tk, tv)]
            ref, size, dots = reference(f64(x[0][r]), front, [np.concatenate(h) for h in held[s]], lens[s], fmt, width ** -0.5)
            assert np.all(np.abs(f64(got[0][r]) - ref) <= attend_tolerance(ref, size, dots, width)), (i, s)
            assert int(got[2][r]) == sample(f64(got[1][r]), float(x[3][r]), 1.0, 20)[0], (i, s)
            r += 1
        lens, held = [after[j] for j in how], [[list(h) for h in held[j]] for j in how]
        for s in range(n):
            assert lens[s] == 0 or same(read(a, s, 0, lens[s]), read(b, s, 0, lens[s])), (i, s)
    assert max(lens) > 20
