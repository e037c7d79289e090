"""How many tokens an entry of a copy between 8-bit caches moves (ad::kv8_copied): tables may say anything, what is moved lies within both caches."""
import ctypes
import itertools

import pytest

from paper_2205_10350_amd import build

I = ctypes.c_int


@pytest.fixture(scope="module")
def copied():
    f = getattr(ctypes.CDLL(build.LIB_PATH), "_ZN2ad10kv8_copiedEiiiiib")   # ad::kv8_copied
    f.restype = I
    f.argtypes = [I] * 5 + [ctypes.c_bool]
    return f


ENDS = [-2 ** 31, -2 ** 31 + 1, -2 ** 31 + 31, -2 ** 30, -33, -1, 0, 1, 31, 32, 33, 50, 63, 64, 96, 97, 100, 300, 2 ** 24, 2 ** 31 - 33, 2 ** 31 - 1]


@pytest.mark.parametrize("closed", [False, True])
@pytest.mark.parametrize("capacity", [1, 31, 32, 33, 100, 300, 1 << 24])
def test_what_is_moved_lies_within_both_caches(copied, capacity, closed):
    for first, end, to, most in itertools.product(sorted({0, min(1, capacity // 32), min(3, capacity // 32), capacity // 32}), ENDS, (1, 32, 50, 100, 1 << 24), (0, 1, 31, 40, 64, 300, 2 ** 31 - 1)):
        got = copied(first, end, capacity, to, most, closed)
        have = max(0, min(end, capacity) - 32 * first)      # (the source's tokens from its block `first` on; numbers without bounds here)
        want = min(have, to, most)
        if not closed and want // 32 < have // 32:          # (the cut's block is complete in the source)
            want -= want % 32
        assert got == want, (first, end, capacity, to, most)
        assert 0 <= got <= min(to, most) and 32 * first + got <= capacity
