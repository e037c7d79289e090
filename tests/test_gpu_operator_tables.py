"""Tables that say something else than there is: nothing beside the rows that a valid sequence owns is written, and those are right.  Outputs lie within larger buffers."""
import pytest

import paper_2205_10350_amd as ad
from test_gpu_kv8_shared import FORMS, Problem, draw, i32, stale, starts

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
