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


def test_copies_of_more_workgroups_than_a_launch_takes_are_refused():
    """Some 270 GB of one head that a single call would move; device pointers are made-up addresses that the refused call does not touch."""
    import paper_2205_10350_amd as ad
    for width, n, capacity in ((128, 257, 1 << 23), (128, 257, 1 << 22), (32, 257, 1 << 24), (64, 129, 1 << 24), (128, 4096, 1 << 24)):
        c = ad.AdKv8Config(n, 1, width, capacity, 1, ad.AD_KV_E4M3, 0)
        at = ctypes.c_void_p(1 << 30)
        assert ad.lib().ad_kv8_copy(ctypes.byref(c), at, ctypes.byref(c), at, at, at, None, at, n, capacity, None) == ad.AD_EINVAL, (width, n, capacity)
        assert "workgroups" in (ad.lib().ad_last_error(None) or b"").decode()
