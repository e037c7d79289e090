"""CPU-only checks of truncated distributions, copies of 8-bit caches and attention over shared texts: refusals of the C ABI (device pointers are made-up addresses that no
refused call may touch) and of the wrappers, and the plain forms that the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2205_10350_amd as ad
from truncate_reference import kept, log_prob_tolerance, sample

P = 1 << 30     # an aligned address
FAR = 1 << 40


def cfg(**kw):
    a = dict(n_seq=2, n_heads=4, head_width=64, capacity=100, k_max=25, format=ad.AD_KV_E4M3, closed=0)
    a.update(kw)
    return ad.AdKv8Config(**a)


def message():
    return (ad.lib().ad_last_error(None) or b"").decode()


def test_sample_tokens_refuses():
    L = ad.lib()

    def go(x=P, dtype=ad.AD_F32, stride=1000, vocab=1000, temp=None, k=None, p=None, q=None, start=None, n_seq=8, u=P, rows=8, tokens=P, log_probs=None):
        return L.ad_sample_tokens(x, dtype, stride, vocab, temp, k, p, q, start, n_seq, u, rows, tokens, log_probs, None)
    for bad in (dict(x=None), dict(x=P + 2), dict(dtype=ad.AD_BF16, x=P + 1), dict(dtype=2), dict(stride=999), dict(vocab=0), dict(vocab=(1 << 24) + 1, stride=1 << 25), dict(u=None),
                dict(tokens=None), dict(rows=-1, n_seq=-1), dict(n_seq=7), dict(start=P, n_seq=0), dict(start=P, n_seq=4097), dict(rows=1 << 22, n_seq=1 << 22)):
        assert go(**bad) == ad.AD_EINVAL, bad
        assert "ad_sample_tokens" in message()
    assert go(rows=0, n_seq=0, x=None, u=None, tokens=None) == ad.AD_OK                # nothing to do


def test_truncate_scores_refuses():
    L = ad.lib()

    def go(x=P, dtype=ad.AD_F32, stride=1000, vocab=1000, start=None, n_seq=8, rows=8, out=FAR, os=1000):
        return L.ad_truncate_scores(x, dtype, stride, vocab, None, None, None, None, start, n_seq, rows, out, os, None)
    for bad in (dict(x=None), dict(out=None), dict(out=FAR + 2), dict(os=999), dict(dtype=3), dict(vocab=-1), dict(n_seq=9), dict(out=P, os=1001), dict(out=P + 4), dict(out=P - 4),
                dict(out=P + 4 * 7999), dict(out=P - 4 * 7999)):
        assert go(**bad) == ad.AD_EINVAL, bad
        assert "ad_truncate_scores" in message()
    assert go(rows=0, n_seq=0) == ad.AD_OK


def test_copy_refuses():
    L = ad.lib()
    c = cfg()
    size = L.ad_kv8_bytes(C.byref(c))

    def go(a=c, origin=P, b=c, cache=FAR, source=P, place=P, begin=None, end=P, n=2, most=100):
        return L.ad_kv8_copy(C.byref(a), origin, C.byref(b), cache, source, place, begin, end, n, most, None)
    for bad in (dict(origin=None), dict(cache=None), dict(origin=P + 128), dict(cache=FAR + 64), dict(source=None), dict(place=None), dict(end=None), dict(n=-1), dict(n=3), dict(most=-1),
                dict(a=cfg(n_heads=2)), dict(a=cfg(head_width=32)), dict(a=cfg(format=ad.AD_KV_I8)), dict(a=cfg(closed=1)), dict(a=cfg(capacity=0)), dict(b=cfg(n_seq=0)),
                dict(cache=P, begin=P), dict(cache=P, a=cfg(capacity=101)), dict(cache=P, a=cfg(k_max=26)), dict(cache=P + size // 256 * 256 - 256), dict(cache=P - 256)):
        assert go(**bad) == ad.AD_EINVAL, bad
        assert message()
    assert go(n=0) == ad.AD_OK and go(most=0) == ad.AD_OK and go(cache=P, n=0) == ad.AD_OK
    assert go(cache=P + (size + 255) // 256 * 256, n=0) == ad.AD_OK                    # (side by side)


def test_attend_shared_refuses():
    L = ad.lib()

    def go(c=cfg(), cache=P, s=cfg(n_seq=3, capacity=2000, closed=1), shared=FAR, q=P, qs=256, heads=4, start=P, length=P, first=P, texts=P, rows=8, most=8, keys=100, together=8,
           text_keys=1000, scale=0.125, out=P, os=256, ws=P, size=1 << 40):
        return L.ad_kv8_attend_shared(C.byref(c), cache, C.byref(s), shared, q, qs, heads, start, length, first, texts, rows, most, keys, together, text_keys, scale, out, os, ws, size, None)
    for bad in (dict(c=cfg(closed=1)), dict(s=cfg(n_heads=2)), dict(s=cfg(head_width=128)), dict(s=cfg(format=ad.AD_KV_I8)), dict(s=cfg(n_seq=0)), dict(cache=None), dict(shared=None),
                dict(shared=FAR + 128), dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 2), dict(qs=252), dict(os=255), dict(heads=6), dict(heads=0), dict(heads=4 * 257),
                dict(start=None), dict(length=None), dict(first=None), dict(texts=None), dict(rows=-1), dict(most=9), dict(together=9), dict(together=-1), dict(most=26, rows=40, together=40),
                dict(keys=-1), dict(text_keys=-1), dict(scale=math.nan), dict(scale=math.inf), dict(ws=None), dict(ws=P + 64)):
        assert go(**bad) == ad.AD_EINVAL, bad
        assert message()
    need = L.ad_kv8_attend_shared_bytes(C.byref(cfg()), C.byref(cfg(n_seq=3, capacity=2000, closed=1)), 4, 8, 100, 1000)
    # 1000 keys of the texts are two splits of 512, the own 100 one: 8 rows x 4 heads x 3 parts of 64 + 2 numbers
    assert need == 8 * 4 * 3 * 64 * 4 + 8 * 4 * 3 * 8
    assert go(size=need - 1) == ad.AD_ENOMEM
    assert L.ad_kv8_attend_shared_bytes(C.byref(cfg()), C.byref(cfg(n_seq=3, capacity=1000)), 4, 8, 100, 1000) == 0       # short texts: one launch
    assert go(rows=0, most=0, together=0) == ad.AD_OK
    wide = cfg(n_seq=1, n_heads=256, k_max=65536, capacity=1 << 17)
    assert go(c=wide, s=wide, heads=65536, qs=65536 * 64, os=65536 * 64, rows=65536, most=65536, together=65536, size=1 << 62) == ad.AD_EINVAL and "workgroups" in message()


def test_wrappers_refuse_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    for call in (lambda x: ad.sample_tokens(x, torch.zeros(2)), ad.truncate_scores):
        for x in (torch.zeros(2, 10), np.zeros((2, 10)), torch.zeros(10), torch.zeros(2, 10, dtype=torch.float64), None):   # (none of them on a GPU)
            with pytest.raises(ad.AdError, match="logits"):
                call(x)


def test_plain_forms():
    x = np.array([math.log(0.1), math.log(0.4), math.log(0.2), math.log(0.3), -math.inf])
    assert kept(x).tolist() == [True, True, True, True, False]
    assert kept(x, k=2).tolist() == [False, True, False, True, False]
    assert kept(x, p=0.65).tolist() == [False, True, False, True, False] and kept(x, p=0.75).tolist() == [False, True, True, True, False]
    assert kept(x, k=3, p=0.75).tolist() == [False, True, False, True, False]            # (0.7 of 0.9)
    assert kept(x, q=0.6).tolist() == [False, True, False, True, False] and kept(x, q=7.0).tolist() == [False, True, False, False, False]
    assert kept(x, p=0.0).tolist() == kept(x, p=-3.0).tolist() == kept(x, k=1).tolist() == [False, True, False, False, False]
    assert kept([1.0, 2.0, 2.0, 2.0], k=2).tolist() == [False, True, True, False]         # equal scores: the lower indices
    assert [sample(x, u)[0] for u in (0.0, 0.09, 0.11, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert sample(x, 0.5, k=2) == (1, pytest.approx(math.log(4 / 7))) and sample(x, 0.6, k=2)[0] == 3
    assert sample([math.nan, 1.0], 0.5)[0] == sample([-math.inf] * 2, 0.5)[0] == sample([1.0, 2.0], 0.5, temperature=0.0)[0] == sample([1.0, 2.0], 0.5, p=math.nan)[0] == -1
    assert log_prob_tolerance(-1.0, 32000) < 1e-6


def test_vocabularies_whose_weights_would_be_too_coarse_are_refused():
    """Weights are 64-bit whole numbers whose sum must fit, too: past 2^20 tokens their rounding could move a sum by more than half a step of an fp32 number below 1."""
    for vocab in ((1 << 20) + 1, 1 << 21, 1 << 24):
        assert ad.lib().ad_sample_tokens(P, ad.AD_F32, vocab, vocab, None, None, None, None, None, 8, P, 8, P, None, None) == ad.AD_EINVAL and "2^20" in message()
        assert ad.lib().ad_truncate_scores(P, ad.AD_BF16, vocab, vocab, None, None, None, None, None, 8, 8, FAR, vocab, None) == ad.AD_EINVAL and "2^20" in message()
    assert ad.lib().ad_sample_tokens(P, ad.AD_F32, 1 << 20, 1 << 20, None, None, None, None, None, 0, P, 0, P, None, None) == ad.AD_OK     # (no rows)
