"""CPU-only checks of the operators without a context: sizes and refusals of the C ABI (device pointers are made-up addresses that no refused
call may touch), and the plain forms that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

import paper_2205_10350_amd as ad
from kv8_reference import accept, attend, held, tokens_as_read

P = 1 << 20     # an aligned address


def cfg(**kw):
    a = dict(n_seq=2, n_heads=4, head_width=64, capacity=100, k_max=25, format=ad.AD_KV_E4M3, closed=0)
    a.update(kw)
    return ad.AdKv8Config(**a)


def message():
    return (ad.lib().ad_last_error(None) or b"").decode()


def test_cache_sizes():
    L = ad.lib()
    c = cfg()
    # 2 x 4 x 4 blocks of 4 KB, their scales (256 bytes), and rings: 25 tokens touch at most 2 blocks, 8 KB each in bf16
    assert L.ad_kv8_bytes(C.byref(c)) == 2 * 4 * (4 * 4096) + 256 + 2 * 4 * 2 * 8192
    c = cfg(closed=1, k_max=0)
    assert L.ad_kv8_bytes(C.byref(c)) == 2 * 4 * (4 * 4096) + 256
    for k_max, ring in ((1, 1), (2, 2), (33, 2), (34, 3)):
        c = cfg(k_max=k_max, n_seq=1, n_heads=1, capacity=32)
        assert L.ad_kv8_bytes(C.byref(c)) == 4096 + 256 + ring * 8192
    big = cfg(n_seq=4096, n_heads=256, capacity=1 << 24, head_width=128)
    assert L.ad_kv8_bytes(C.byref(big)) > 1 << 50


@pytest.mark.parametrize("bad", [dict(n_seq=0), dict(n_seq=4097), dict(n_heads=0), dict(n_heads=257), dict(head_width=48), dict(head_width=16),
                                 dict(capacity=0), dict(capacity=(1 << 24) + 1), dict(k_max=0), dict(k_max=65537), dict(format=2), dict(format=-1), dict(closed=2)])
def test_cache_descriptions_refused(bad):
    L = ad.lib()
    c = cfg(**bad)
    assert L.ad_kv8_check(C.byref(c)) == ad.AD_EINVAL and message()
    assert L.ad_kv8_bytes(C.byref(c)) == 0
    assert L.ad_kv8_attend_bytes(C.byref(c), 4, 10, 100) == 0
    assert L.ad_kv8_append(C.byref(c), P, P, 256, P, 256, P, P, 4, 4, None) == ad.AD_EINVAL
    assert L.ad_kv8_check(None) == ad.AD_EINVAL


def test_append_read_and_attend_refuse():
    L = ad.lib()
    c = C.byref(cfg())

    def append(cache=P, k=P, ks=256, v=P, vs=256, start=P, length=P, rows=8, most=8, c=c):
        return L.ad_kv8_append(c, cache, k, ks, v, vs, start, length, rows, most, None)
    for bad in (dict(cache=None), dict(cache=P + 16), dict(k=None), dict(v=None), dict(start=None), dict(length=None), dict(k=P + 8), dict(v=P + 2),
                dict(ks=255), dict(vs=248), dict(ks=260), dict(rows=-1), dict(most=9), dict(most=-1), dict(rows=40, most=26)):
        assert append(**bad) == ad.AD_EINVAL, bad
        assert message()
    assert append(rows=200, most=101, c=C.byref(cfg(closed=1))) == ad.AD_EINVAL
    assert append(rows=0, most=0) == ad.AD_OK and append(most=0) == ad.AD_OK          # nothing to do

    def read(cache=P, start=P, begin=P, length=P, rows=8, most=8, dtype=ad.AD_BF16, k=P, v=P):
        return L.ad_kv8_read(c, cache, start, begin, length, rows, most, dtype, k, v, None)
    for bad in (dict(cache=None), dict(start=None), dict(begin=None), dict(length=None), dict(k=None), dict(v=P + 8), dict(dtype=2), dict(most=9), dict(rows=-1)):
        assert read(**bad) == ad.AD_EINVAL, bad
    assert read(rows=0, most=0) == ad.AD_OK

    def go(cache=P, q=P, qs=256, heads=4, start=P, length=P, rows=8, most=8, keys=100, scale=0.125, out=P, os=256, ws=P, size=1 << 30, c=c):
        return L.ad_kv8_attend(c, cache, q, qs, heads, start, length, rows, most, keys, scale, out, os, ws, size, None)
    for bad in (dict(cache=None), dict(cache=P + 128), dict(q=None), dict(out=None), dict(q=P + 4), dict(out=P + 8), dict(qs=252), dict(os=100), dict(heads=6),
                dict(heads=2), dict(heads=0), dict(heads=4 * 257), dict(rows=-1), dict(most=9), dict(rows=40, most=26), dict(keys=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(start=None), dict(length=None)):
        assert go(**bad) == ad.AD_EINVAL, bad
    assert go(rows=0, most=0) == ad.AD_OK
    long = C.byref(cfg(capacity=100000))
    need = L.ad_kv8_attend_bytes(long, 4, 8, 100000)
    assert need > 0 and L.ad_kv8_attend_bytes(long, 4, 8, 200) == 0
    assert go(c=long, keys=100000, size=need - 1) == ad.AD_ENOMEM
    assert go(c=long, keys=100000, ws=None, size=need) == ad.AD_EINVAL
    assert go(c=long, keys=100000, ws=P + 64, size=need) == ad.AD_EINVAL
    # more workgroups than a launch takes: 65,536 heads x 65,536 rows; the joined rows of 2^26 (row, head) pairs
    wide = C.byref(cfg(n_seq=1, n_heads=256, k_max=65536, capacity=1 << 17))
    assert go(c=wide, heads=65536, qs=65536 * 64, os=65536 * 64, rows=65536, most=65536, keys=1000, size=1 << 62) == ad.AD_EINVAL and "workgroups" in message()
    assert go(c=wide, heads=1024, qs=65536, os=65536, rows=65536, most=65536, keys=1 << 17, size=1 << 62) == ad.AD_EINVAL and "workgroups" in message()


def test_accept_sampled_refuses():
    L = ad.lib()

    def go(x=P, dtype=ad.AD_F32, stride=1000, vocab=1000, draft=P, probs=None, ps=1000, temp=None, u=P, v=P, start=P, n_seq=2, rows=8, most=8, n=P, tok=P,
           ws=P, size=1 << 30):
        return L.ad_accept_sampled(x, dtype, stride, vocab, draft, probs, ps, temp, u, v, start, n_seq, rows, most, n, tok, ws, size, None)
    for bad in (dict(x=None), dict(x=P + 2), dict(dtype=2), dict(stride=999), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(draft=None), dict(probs=P, ps=999),
                dict(u=None), dict(v=None), dict(start=None), dict(n_seq=0), dict(n_seq=4097), dict(rows=0), dict(most=0), dict(most=9), dict(rows=70000, most=65536),
                dict(n=None), dict(tok=None), dict(ws=None), dict(ws=P + 8)):
        assert go(**bad) == ad.AD_EINVAL, bad
        assert message()
    need = L.ad_accept_sampled_bytes(2, 8, 1000)
    assert need > 0 and go(size=need - 1) == ad.AD_ENOMEM
    assert L.ad_accept_sampled_bytes(0, 8, 1000) == 0 and L.ad_accept_sampled_bytes(2, 0, 1000) == 0 and L.ad_accept_sampled_bytes(2, 8, 0) == 0


def test_wrappers_refuse_tensors_that_do_not_fit():
    torch = pytest.importorskip("torch")
    with pytest.raises(ad.AdError):
        ad.Kv8Cache(1, 4, 64, 100, format="fp4", device="cuda:0")
    with pytest.raises(ad.AdError, match="GPU"):
        ad.Kv8Cache(1, 4, 64, 100, device="cpu")
    with pytest.raises(ad.AdError, match="32-bit"):
        ad.Kv8Cache(1, 4, 64, (1 << 32) + 100, device="cuda:0")
    with pytest.raises(ad.AdError):
        ad.accept_sampled(torch.zeros(2, 10), None, None, None, None)      # not on a GPU
    with pytest.raises(ad.AdError):
        ad.accept_sampled(np.zeros((2, 10)), None, None, None, None)


def test_plain_forms():
    """The reference itself: known values, and the property that a row's own block is as it was written."""
    x = np.zeros((32, 4))
    x[0] = [448, 447, 17, 0.001]
    assert held(x, "e4m3")[0].tolist() == [448, 448, 16, 0.001953125]      # 17: halfway to 18, to even; 0.001 is above half of the least step, 2^-9
    x[0] = [127, 63.5, 0.5, 1.5]
    assert held(x, "i8")[0].tolist() == [127, 64, 0, 2]                                               # ties to even
    rng = np.random.default_rng(0)
    t = rng.standard_normal((70, 2, 8))
    read = tokens_as_read(t, 69, "i8")
    assert (read[64:] == t[64:]).all() and (read[:64] != t[:64]).any()
    out, size, _ = attend(rng.standard_normal((4, 8)), t, t, 69, "i8", 0.3)
    assert out.shape == (4, 8) and (np.abs(out) <= size + 1e-12).all()
    p = np.log(np.array([[0.5, 0.25, 0.25]]))
    assert accept(p, [0], None, 1.0, [0.49], 0.0) == [0] and accept(p, [0], None, 1.0, [0.51], 0.49) == [1] and accept(p, [0], None, 1.0, [0.51], 0.51) == [2]
    q = np.array([[0.25, 0.5, 0.25]])
    assert accept(p, [1], q, 1.0, [0.49], 0.0) == [1] and accept(p, [1], q, 1.0, [0.51], 0.9) == [0]
    assert accept(p, [ad.AD_NEVER], None, 1.0, [0.0], 0.6) == [1]


def config(name="tiny", dtype="bf16_kv_i8", **kw):
    from ad_inputs import SPECIAL, model_dims
    a = dict(max_batch=2, max_src=24, max_len=32, k_max=8, special=SPECIAL)
    a.update(kw)
    return ad.make_config(model_dims(name) if isinstance(name, str) else name, dtype=dtype, **a)


def test_contexts_with_caches_in_8_bits():
    """Same weights as bf16; smaller workspaces once outputs are long; longer outputs than bf16 rows allow, but not beside a drafter."""
    for dtype in ("bf16_kv_e4m3", "bf16_kv_i8"):
        assert ad.config_check(config(dtype=dtype)) == ad.AD_OK
        assert ad.weights_layout(config(dtype=dtype)) == ad.weights_layout(config(dtype="bf16"))
        assert ad.weights_layout(config(dtype=dtype, tie_output=True)) == ad.weights_layout(config(dtype="bf16", tie_output=True))
        big = dict(max_batch=32, max_src=500, max_len=400, k_max=16)
        small, wide = (ad.workspace_bytes(config("big", dtype=t, **big), False) for t in (dtype, "bf16"))
        caches = 6 * 2 * 32 * (500 + 416) * 1024 * 2
        assert wide - small > 0.4 * caches
        assert ad.config_check(config("base", dtype=dtype, max_len=8000)) == ad.AD_OK
        assert ad.config_check(config("base", dtype="bf16", max_len=8000)) == ad.AD_EINVAL
        assert ad.workspace_bytes(config("base", dtype=dtype, max_len=8000), False) > 0
        assert ad.workspace_bytes(config("base", dtype=dtype, max_len=8000), True) == 0 and "drafter" in message()
        assert ad.workspace_bytes(config("base", dtype=dtype), True) > 0
        assert ad.config_check(config("micro", dtype=dtype)) == ad.AD_EINVAL and "head size" in message()      # heads of 16
        assert ad.config_check(config("base", dtype=dtype, max_src=8000)) == ad.AD_EINVAL                       # the encoder's own attention


def test_verify_sampled_without_a_context():
    assert ad.lib().ad_verify_sampled(None, None, None, None, None, None, None, None, None) == ad.AD_EINVAL


def test_accept_sampled_takes_as_many_rows_as_it_can_look_up():
    """max_rows above 65,535 is refused where rows go by sequence only."""
    L = ad.lib()

    def go(n_seq, rows, most, ws=None, size=0):
        return L.ad_accept_sampled(P, ad.AD_F32, 1000, 1000, P, None, 1000, None, P, P, P, n_seq, rows, most, P, P, ws, size, None)
    assert go(4, 70000, 70000) == ad.AD_EINVAL and "65535" in message()
    assert go(5, 70000, 70000) == ad.AD_EINVAL and "null" in message()               # (looked up: the next thing that is wrong)
    assert go(5, 70000, 70000, ws=P) == ad.AD_ENOMEM


def test_accept_sampled_of_no_rows_needs_no_more_than_the_counts_place():
    L = ad.lib()

    def go(rows=0, most=0, u=P, start=P, n=P):
        return L.ad_accept_sampled(None, ad.AD_F32, 1000, 1000, None, None, 1000, None, None, u, start, 3, rows, most, n, None, None, 0, None)
    for bad in (dict(most=1), dict(rows=-1, most=-1), dict(u=None), dict(start=None), dict(n=None), dict(rows=1, most=1)):
        assert go(**bad) == ad.AD_EINVAL, bad


@pytest.mark.parametrize("dtype", ["bf16_kv_e4m", "BF16", "i8", None, 0])
def test_unknown_dtypes_of_contexts_are_refused(dtype):
    with pytest.raises(ad.AdError, match="dtype") as e:
        config(dtype=dtype)
    assert e.value.code == ad.AD_EINVAL
