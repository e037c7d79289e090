"""Where copies of 8-bit caches end: inside a block of the source, with nothing, outside the caches."""
import numpy as np
import pytest

import paper_2205_10350_amd as ad

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

HEADS, WIDTH, CAPACITY = 2, 32, 320


def i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def starts(n):
    return i32(np.concatenate(([0], np.cumsum(n))))


def tokens(seed, n=CAPACITY):
    return [torch.tensor(np.random.default_rng(seed + i).standard_normal((n, HEADS, WIDTH)), dtype=torch.float32).to(torch.bfloat16).cuda() for i in range(2)]


def make(n_seq=2, **kw):
    cache = ad.Kv8Cache(n_seq, HEADS, WIDTH, **dict(dict(capacity=CAPACITY, k_max=7), **kw))
    cache.memory.fill_(0xFF)   # (whatever lies there must not matter: NaN patterns of every type)
    return cache


def feed(cache, seq, kv, begin, end):
    """Tokens begin .. end - 1 of kv = k, v become those of the sequence, k_max at a time (closed: at once)."""
    step = cache.cfg.capacity if cache.cfg.closed else cache.cfg.k_max
    for at in range(begin, end, step):
        rows = [min(end - at, step) if b == seq else 0 for b in range(cache.cfg.n_seq)]
        cache.append(*(t[at:at + step][:rows[seq]].contiguous() for t in kv), starts(rows), i32([at] * len(rows)))


def read(cache, seq, begin, end):
    rows = [end - begin if b == seq else 0 for b in range(cache.cfg.n_seq)]
    return torch.stack(cache.read(starts(rows), i32([begin] * len(rows)), i32([end] * len(rows)), rows=end - begin, dtype=torch.float32)).view(torch.int32)


# tokens of the source, its k_max, the first token, capacity and max_tokens of the copy, tokens that it has
CUT = [(300, 1, 0, 50, None, 32), (200, 1, 0, 100, 100, 96), (200, 7, 0, 100, 100, 96), (300, 1, 0, CAPACITY, 40, 32), (300, 60, 0, CAPACITY, 31, 0), (300, 7, 0, 100, 70, 64),
       (300, 1, 64, 50, None, 32), (256, 1, 0, 50, None, 32), (300, 60, 0, CAPACITY, 287, 256),
       # (not cut, or in the incomplete block, which the source holds in bf16: that goes with it)
       (300, 7, 256, CAPACITY, 43, 43), (300, 7, 0, CAPACITY, 299, 299), (300, 1, 0, 289, None, 289), (300, 7, 0, CAPACITY, 288, 288),
       (300, 1, 0, 300, None, 300), (300, 7, 0, CAPACITY, 300, 300), (300, 1, 256, 50, 44, 44), (50, 7, 0, 50, 50, 50)]


@pytest.mark.parametrize("fmt", ["e4m3", "i8"])
@pytest.mark.parametrize("n,k_max,begin,capacity,most,has", CUT)
def test_a_copy_cut_short_ends_with_a_whole_block(n, k_max, begin, capacity, most, has, fmt):
    """A block that a cut lies in is left out where it is complete in the source, which holds it in 8 bits alone."""
    kv = tokens(n + k_max)
    origin = make(k_max=k_max, format=fmt)
    feed(origin, 1, kv, 0, n)
    got, want = (make(3, capacity=capacity, format=fmt) for _ in range(2))
    first = None if begin == 0 else i32([begin])
    got.copy(i32([1]), i32([2]), i32([n]), begin=first, origin=origin, max_tokens=most)
    want.copy(i32([1]), i32([2]), i32([begin + has]), begin=first, origin=origin)
    assert torch.equal(got.memory, want.memory)
    whole = has // 32 * 32
    assert torch.equal(read(got, 2, 0, whole), read(origin, 1, begin, begin + whole))
    # what follows: as if all of it had been written there
    other = make(3, capacity=capacity, format=fmt)
    mine = [t[begin:] for t in kv]
    feed(other, 2, mine, 0, has)
    end = min(has + 40, capacity, CAPACITY - begin)
    for cache in (got, other):
        feed(cache, 2, mine, has, end)
    assert torch.equal(read(got, 2, 0, end), read(other, 2, 0, end))


def test_a_fork_cut_short_and_others_that_are_not():
    kv = tokens(1)
    got, want = (make(6, k_max=60) for _ in range(2))
    for cache in (got, want):
        for b, n in enumerate((300, 40, 64)):
            feed(cache, b, kv, 0, n)
    got.copy(i32([0, 1, 2]), i32([3, 4, 5]), i32([300, 40, 64]), max_tokens=45)
    want.copy(i32([0, 1, 2]), i32([3, 4, 5]), i32([32, 40, 32]))
    assert torch.equal(got.memory, want.memory)


def test_a_closed_copy_is_cut_anywhere():
    kv = tokens(2)
    origin = make(closed=True)
    feed(origin, 1, kv, 0, 300)
    for capacity, most, has in ((50, None, 50), (320, 45, 45), (33, 40, 33)):
        got = make(closed=True, capacity=capacity)
        got.copy(i32([1]), i32([0]), i32([300]), origin=origin, max_tokens=most)
        assert torch.equal(read(got, 0, 0, has), read(origin, 1, 0, has))


def test_ends_and_begins_that_are_no_lengths():
    """Ends far below 0 with begins above it, on both sides of what 32 bits hold: nothing is moved."""
    kv = tokens(3, 100)
    origin, cache = make(capacity=100), make(capacity=100)
    for b in range(2):
        feed(origin, b, kv, 0, 100)
        feed(cache, b, kv, 0, 70)
    before = cache.memory.clone()
    for end, begin in ((-2 ** 31, 32), (-2 ** 31, 96), (-2 ** 31 + 31, 32), (-2 ** 31 + 95, 2 ** 31 - 1), (-2 ** 31, -2 ** 31), (-1, 64), (0, 32), (31, 32), (32, 32)):
        cache.copy(i32([0, 1]), i32([1, 0]), i32([end, end]), begin=i32([begin, begin]), origin=origin)
        assert torch.equal(cache.memory, before), (end, begin)


def test_of_entries_with_one_place_the_first_counts_without_tokens_too():
    kv = tokens(4, 100)
    got, want = (make(6, capacity=100, k_max=100) for _ in range(2))
    for cache in (got, want):
        for b, n in enumerate((100, 40, 64)):
            feed(cache, b, kv, 0, n)
    got.copy(i32([0, 1, 2, 1]), i32([3, 3, 4, 4]), i32([0, 40, 64, 40]))
    want.copy(i32([2]), i32([4]), i32([64]))
    assert torch.equal(got.memory, want.memory)
    # an entry of a sequence or place that is not there is none
    got.copy(i32([9, 1, -1, 2]), i32([3, 3, 5, 5]), i32([0, 40, 40, 64]))
    want.copy(i32([1, 2]), i32([3, 5]), i32([40, 64]))
    assert torch.equal(got.memory, want.memory)
    # nor does one that begins behind its end, from another cache, leave its place to the next
    other = make(6, capacity=100)
    before = other.memory.clone()
    other.copy(i32([0, 1]), i32([3, 3]), i32([64, 40]), begin=i32([64, 0]), origin=got)
    assert torch.equal(other.memory, before)
