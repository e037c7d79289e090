"""Contexts whose caches are in 8 bits, and block verification for sampled decoding: whole decodes through the C ABI."""
import numpy as np
import pytest

import paper_2205_10350_amd as ad
from ad_inputs import SPECIAL, edit_guide, init_weights, model_dims, positional_draft
import kv8_oracle as K
from kv8_reference import accept, tokens_as_read
from oracle import ad_oracle as O

pytestmark = pytest.mark.gpu
EOS = SPECIAL["eos"]


def context(dims, w, dtype, B=3, max_src=40, max_len=48, k_max=24, logits=False, drafter=None):
    cfg = ad.make_config(dims, max_batch=B, max_src=max_src, max_len=max_len, k_max=k_max, dtype=dtype, special=SPECIAL, debug_logits=logits)
    return ad.Context(cfg, w, drafter)


def sources(dims, lens, seed=3):
    rng = np.random.default_rng(seed)
    return [rng.integers(5, dims["vocab"], size=n).astype(np.int32) for n in lens]


@pytest.mark.parametrize("dtype", ["bf16_kv_e4m3", "bf16_kv_i8"])
@pytest.mark.parametrize("name,std", [("tiny", 0.15), ("wide_head", 0.1), ("base", 0.02)])
def test_decodes_agree_token_for_token(name, std, dtype):
    dims = model_dims(name)
    w = init_weights(dims, 21, std)
    srcs = sources(dims, [40, 1, 33])
    with context(dims, w, dtype) as ctx:
        greedy, st = ctx.decode_greedy(srcs)
        guides = [edit_guide(g, 0.2, 5 + b, dims["vocab"]) for b, g in enumerate(greedy)]
        drafts = [positional_draft(g, 0.2, 6 + b, dims["vocab"])[0] for b, g in enumerate(greedy)]
        for _ in range(2):      # (the second time over: shapes come back, graphs are replayed)
            iad, st1 = ctx.decode_iad(srcs, guides)
            gad, st2 = ctx.decode_gad(srcs, 20, draft_override=drafts)
            assert iad == greedy and gad == greedy
            assert st2["iterations"] < st["iterations"]
        for b in (0, 2):
            assert ctx.decode_greedy(srcs[b:b + 1])[0] == greedy[b:b + 1]
        ctx.set_option(ad.AD_OPT_GRAPHS, 0)
        assert ctx.decode_gad(srcs, 20, draft_override=drafts)[0] == greedy
        ctx.encode(ad.AD_VERIFIER, srcs)
        n, nx = ctx.verify([g[:5] for g in greedy], static=True)
        assert n.tolist() == [min(5, len(g)) for g in greedy]


@pytest.mark.parametrize("dtype", ["bf16_kv_e4m3", "bf16_kv_i8"])
def test_a_rows_scores_do_not_depend_on_its_block(dtype):
    dims = model_dims("tiny")
    w = init_weights(dims, 22, 0.15)
    srcs = sources(dims, [30, 12])
    tok = sources(dims, [46, 46], seed=9)
    with context(dims, w, dtype, B=2, logits=True, max_len=64, k_max=46) as ctx:
        rows = {}
        ctx.encode(ad.AD_VERIFIER, srcs)
        n, nx, ver = ctx.verify([t.tolist() for t in tok], want_verified=True)
        all_at_once = ctx.debug_logits().reshape(2, 46, -1)
        # the greedy continuation, fed one by one and in blocks: same scores where the fed tokens are the same
        greedy, _ = ctx.decode_greedy(srcs)
        L = min(len(g) for g in greedy)
        for step in (1, 5, 40):
            ctx.encode(ad.AD_VERIFIER, srcs)
            got, at = [], 0
            while at < L:
                m = min(step, L - at)
                ctx.verify([g[at:at + m] for g in greedy])
                got.append(ctx.debug_logits().reshape(2, m, -1))
                at += m
            rows[step] = np.concatenate(got, 1)
        assert np.array_equal(rows[1], rows[5]) and np.array_equal(rows[1], rows[40])
        assert np.array_equal(rows[1][:, 0], all_at_once[:, 0])


class HeldOracle(O.Model):
    """The oracle with the decoder's keys and values as an 8-bit cache holds them (bf16 rows first)."""
    fmt, deciding = "e4m3", False

    def decode_full(self, memory, tokens, causal=True):
        self.deciding = True
        try:
            return super().decode_full(memory, tokens, causal)
        finally:
            self.deciding = False

    def attention(self, q, k, v, vis):
        if not self.deciding:
            return super().attention(q, k, v, vis)
        closed = vis[0] == vis[-1] and len(vis) > 1
        heads = lambda t: O.bf16_round(t).reshape(len(t), self.H, self.dh)
        k, v = heads(k), heads(v)
        out = []
        for i in range(len(q)):
            kk, vv = (tokens_as_read(t[:vis[i]], i, self.fmt, closed).reshape(-1, self.d) for t in (k, v))
            out.append(super().attention(q[i:i + 1], kk, vv, [vis[i]])[0])
        return np.stack(out)


@pytest.mark.parametrize("dtype", ["bf16_kv_e4m3", "bf16_kv_i8"])
def test_scores_against_the_oracle_over_held_keys_and_values(dtype):
    """The bf16 contract's 2e-2, and what its roundings move across a step of a held value: at weights of N(0, 0.02) and width 128 an attention sublayer's output has
    values of 0.05 beside the rows' 1; a step moves a value by up to 2^-3, four sublayers add up as independent: 4^0.5 * 0.05 * 2^-3 = 0.0125 of a row,
    0.23 of that in a score's rms, and five times that at most among 2000 * 40 scores: 1.5e-2."""
    dims = model_dims("tiny")
    w = init_weights(dims, 23, 0.02)
    src = sources(dims, [37])
    tok = sources(dims, [40], seed=10)[0].tolist()
    m = HeldOracle(dims, {n: (O.bf16_round(a) if a.ndim == 2 else a) for n, a in w.items()}, np.float64, max_pos=128)
    m.fmt = dtype[8:]
    want = m.decode_full(m.encode(src[0]), [SPECIAL["bos"]] + tok[:39])
    with context(dims, w, dtype, B=1, logits=True, k_max=40) as ctx:
        ctx.encode(ad.AD_VERIFIER, src)
        ctx.verify([tok])
        assert np.abs(ctx.debug_logits() - want).max() < 2e-2 + 1.5e-2


def test_encoder_teams_that_give_up_leave_the_memory_right():
    """A team wait of nothing: the encoder's launch is given up, and the call that finds out encodes again, memory in 8 bits included."""
    dims = model_dims("base")
    w = init_weights(dims, 33)
    srcs = sources(dims, [25, 7])
    got = []
    for wait in (None, 0):
        with context(dims, w, "bf16_kv_e4m3", B=2) as ctx:
            if wait is not None:
                ctx.set_option(ad.AD_OPT_TEAM_WAIT, wait)
            got.append(ctx.decode_greedy(srcs)[0])
            if wait is not None:
                assert ctx.get_option(ad.AD_OPT_TEAM_FAILURES) > 0
    assert got[0] == got[1]


def test_outputs_longer_than_rows_of_bf16_allow():
    """700 tokens of a head of width 64 (bf16 rows: at most 526 with the block), over several splits of the keys."""
    dims = dict(enc_layers=1, dec_layers=2, d_model=128, n_heads=2, d_ffn=256, vocab=2000)
    w = init_weights(dims, 24, 0.1)
    w["out.w"][EOS] = 0      # (an end of sentence that never scores highest)
    srcs = sources(dims, [20, 31])
    bf16 = ad.make_config(dims, max_batch=2, max_src=40, max_len=700, k_max=64, dtype="bf16", special=SPECIAL)
    assert ad.config_check(bf16) == ad.AD_EINVAL
    with context(dims, w, "bf16_kv_i8", B=2, max_len=700, k_max=64) as ctx:
        greedy, st = ctx.decode_greedy(srcs)
        assert max(len(g) for g in greedy) > 600
        drafts = [positional_draft(g, 0.05, 6 + b, dims["vocab"])[0] for b, g in enumerate(greedy)]
        gad, st2 = ctx.decode_gad(srcs, 64, draft_override=drafts)
        assert gad == greedy and st2["iterations"] < st["iterations"] / 4


def test_timing_a_forward_leaves_the_caches_as_they_were():
    dims = model_dims("tiny")
    w = init_weights(dims, 25, 0.15)
    srcs = sources(dims, [30, 12])
    with context(dims, w, "bf16_kv_e4m3", B=2, max_len=64, k_max=40) as ctx:
        greedy, _ = ctx.decode_greedy(srcs)
        L = min(len(g) for g in greedy)
        ctx.encode(ad.AD_VERIFIER, srcs)
        at = 0
        while at < L:
            m = min(7, L - at)
            # the drafted block agrees for m tokens; what follows is rejected, and its rows are timed over and over
            n, _ = ctx.verify([g[at:at + m] + ([ad.AD_NEVER] if at + m < L else []) for g in greedy])
            ctx.time_verify_forward(reps=2)
            at += int(n.min())
            assert n.tolist() == [int(n[0])] * 2
        assert all(o == g[:len(o)] for o, g in zip(ctx.output(), greedy))


def sampled_decode(ctx, srcs, guides, rng, temperature, vocab, max_len):
    """A whole sampled decode in blocks; every call's tokens are checked against the plain form over the call's own scores."""
    B = len(srcs)
    ctx.encode(ad.AD_VERIFIER, srcs)
    out, done = [[] for _ in range(B)], [False] * B
    calls = 0
    while not all(done):
        drafts = []
        for b in range(B):
            d = [] if done[b] else guides[b][len(out[b]):len(out[b]) + 12] or [ad.AD_NEVER]
            drafts.append(d[:max_len - len(out[b])])
        u = [rng.random(len(d)).astype(np.float32) for d in drafts]
        v = rng.random(B).astype(np.float32)
        n, nx, ver = ctx.verify_sampled(drafts, u, v, temperature, want_verified=True)
        scores, r = ctx.debug_logits(), 0
        for b, d in enumerate(drafts):
            if not d:
                assert n[b] == 0
                continue
            want = accept(scores[r:r + len(d)], d, None, temperature[b], u[b], v[b])
            if EOS in want:
                want = want[:want.index(EOS) + 1]
            r += len(d)
            assert ver[b, :len(want)].tolist() == want and n[b] == len(want) and nx[b] == want[-1]
            out[b] += want
            done[b] = want[-1] == EOS or len(out[b]) >= max_len
        calls += 1
    assert ctx.output() == out
    return out, calls


@pytest.mark.parametrize("name,dtype,std", [("tiny", "fp32", 0.15), ("tiny", "bf16", 0.15), ("tiny", "bf16_kv_i8", 0.15), ("base", "bf16", 0.02),
                                            ("base", "bf16_kv_e4m3", 0.02)])
def test_sampled_decodes_in_blocks(name, dtype, std):
    dims = model_dims(name)
    w = init_weights(dims, 26, std)
    srcs = sources(dims, [25, 7, 18])
    with context(dims, w, dtype, logits=True) as ctx:
        greedy, _ = ctx.decode_greedy(srcs)
        rng = np.random.default_rng(27)
        # cold, lukewarm and hot: guides nearly always stand, sometimes, hardly ever
        for _ in range(3):
            out, calls = sampled_decode(ctx, srcs, greedy, rng, np.array([0.02, 0.2, 1.0], np.float32), dims["vocab"], 48)
        assert calls <= 48
        # greedy verification afterwards is what it was
        assert ctx.decode_greedy(srcs)[0] == greedy


def test_sampled_verification_of_drafts_from_the_block_drafter_and_teams_that_give_up():
    """A run as a user makes it: caches in 8 bits for the verifier, a drafter beside it, blocks drafted and verified from random numbers; then the
    bf16 context with a team wait of nothing, whose launches are all repeated: same tokens as without teams."""
    dims = model_dims("base")
    w, wd = init_weights(dims, 28), init_weights(dims, 29)
    srcs = sources(dims, [25, 7])
    with context(dims, w, "bf16_kv_e4m3", B=2, logits=True, drafter=wd) as ctx:
        rng = np.random.default_rng(30)
        ctx.encode(ad.AD_VERIFIER, srcs)
        ctx.encode(ad.AD_DRAFTER, srcs)
        out = [[], []]
        for _ in range(6):
            drafts = [d.tolist() for d in ctx.draft_nat(6)]
            u, v = rng.random((2, 6)).astype(np.float32), rng.random(2).astype(np.float32)
            n, nx, ver = ctx.verify_sampled(drafts, u, v, 0.05, want_verified=True)
            s = ctx.debug_logits()
            for b in range(2):
                want = accept(s[6 * b:6 * b + 6], drafts[b], None, np.float32(0.05), u[b], v[b])
                want = want[:want.index(EOS) + 1] if EOS in want else want
                assert ver[b, :len(want)].tolist() == want and n[b] == len(want)
                out[b] += want
            if any(o[-1] == EOS for o in out):
                break
        assert ctx.output() == out
    drafts = [list(range(5, 15)), list(range(20, 28))]
    rng = np.random.default_rng(31)
    u, v = rng.random((2, 10)).astype(np.float32), rng.random(2).astype(np.float32)
    got = []
    for teams, wait in ((0, None), (1, None), (1, 0)):
        with context(dims, w, "bf16", B=2, logits=True) as ctx:
            ctx.set_option(ad.AD_OPT_TEAMS, teams)
            if wait is not None:
                ctx.set_option(ad.AD_OPT_TEAM_WAIT, wait)
            ctx.encode(ad.AD_VERIFIER, srcs)
            for _ in range(2):
                ctx.verify_sampled(drafts, u, v, 3.0)
            got.append(ctx.output())
            if wait == 0:
                assert ctx.get_option(ad.AD_OPT_TEAM_FAILURES) > 0
    assert got[0] == got[1] == got[2]


def test_sampled_verification_refuses():
    dims = model_dims("tiny")
    w = init_weights(dims, 32, 0.15)
    srcs = sources(dims, [9])
    with context(dims, w, "bf16", B=1) as ctx:
        ctx.encode(ad.AD_VERIFIER, srcs)
        with pytest.raises(ad.AdError) as e:
            ctx.verify_sampled([[5]], [[0.5]], [0.5])
        assert e.value.code == ad.AD_ESTATE
    with context(dims, w, "bf16", B=1, logits=True) as ctx:
        with pytest.raises(ad.AdError) as e:
            ctx.B = 1
            ctx.verify_sampled([[5]], [[0.5]], [0.5])
        assert e.value.code == ad.AD_ESTATE
        ctx.encode(ad.AD_VERIFIER, srcs)
        for u, v, t in (([[1.0]], [0.5], None), ([[-0.1]], [0.5], None), ([[float("nan")]], [0.5], None), ([[0.5]], [1.0], None), ([[0.5]], [0.5], 0.0),
                        ([[0.5]], [0.5], float("inf")), ([[0.5]], [0.5], float("nan")), ([[]], [0.5], None), ([[0.5]], [0.5, 0.5], None)):
            with pytest.raises(ad.AdError) as e:
                ctx.verify_sampled([[5]], u, v, t)
            assert e.value.code == ad.AD_EINVAL
        ctx.set_gadpp(3, 1.0)
        with pytest.raises(ad.AdError) as e:
            ctx.verify_sampled([[5]], [[0.5]], [0.5])
        assert e.value.code == ad.AD_ESTATE
        ctx.set_gadpp(1, 0.0)
        n, _ = ctx.verify_sampled([[5]], [[0.5]], [0.5])      # and the context is as it was
        assert n.tolist() == [1]


@pytest.mark.parametrize("model", K.MODELS)
def test_scores_of_peaked_attention_against_the_oracle_over_held_keys_and_values(model):
    """Models in which wrong keys, scales, blocks or caches that are not held in 8 bits move the scores well past the tolerance (test_kv8_oracle.py shows it)."""
    fmt = model[0]
    dims, w, src, tok = K.problem(*model)
    want, tol = K.tolerance(fmt, dims, w, src, tok)
    with context(dims, w, "bf16_kv_" + fmt, B=1, max_src=K.S, max_len=K.T, k_max=K.T, logits=True) as ctx:
        ctx.encode(ad.AD_VERIFIER, [src])
        ctx.verify([tok])
        assert K.far(ctx.debug_logits(), want) <= tol, K.far(ctx.debug_logits(), want) / tol


@pytest.mark.parametrize("dtype", ["bf16_kv_e4m3", "bf16_kv_i8"])
def test_ragged_batches_of_many_sequences(dtype):
    """40 sequences, one long source and one long output among short ones and finished ones: writes, tiles and joins of rows go by the table of packed rows there, over two
    splits of the keys.  Each sequence's scores are bit for bit those that it has by itself, where they go by sequence."""
    dims = dict(enc_layers=1, dec_layers=2, d_model=128, n_heads=4, d_ffn=256, vocab=512)
    w = init_weights(dims, 34, 0.1)
    w["out.w"][EOS] = 0      # (an end of sentence that never scores highest)
    n_seq, long, step = 40, 1300, 300
    srcs = sources(dims, [700 if b == 3 else 1 + b % 3 for b in range(n_seq)], seed=35)
    most = [long if b == 5 else 1 + b % 4 for b in range(n_seq)]
    rng = np.random.default_rng(36)
    with context(dims, w, dtype, B=n_seq, max_src=800, max_len=long, k_max=step, logits=True) as ctx:
        greedy = ctx.decode_greedy([srcs[5]], max_out=[long])[0][0]
        assert len(greedy) == long

        def decode(which, drafts=None):
            """All drafts of a run, per call, and every sequence's scores."""
            ctx.encode(ad.AD_VERIFIER, [srcs[b] for b in which], max_out=[most[b] for b in which])
            done, used, got = [0] * len(which), [], [[] for _ in which]
            while done[which.index(5)] < long if 5 in which else any(d < most[b] for d, b in zip(done, which)):
                d = []
                for i, b in enumerate(which):
                    if drafts is not None:
                        d.append(drafts[len(used)][b])
                    elif b == 5:
                        d.append(greedy[done[i]:done[i] + step])
                    else:
                        d.append(rng.integers(5, 512, size=int(rng.integers(1, 4))).tolist() if done[i] < most[b] else [])
                n, _ = ctx.verify(d)
                s, at = ctx.debug_logits(), 0
                for i in range(len(which)):
                    got[i].append(s[at:at + len(d[i])])
                    at += len(d[i])
                    done[i] += int(n[i])
                used.append({b: x for b, x in zip(which, d)})
            return used, [np.concatenate(x) for x in got]
        drafts, together = decode(list(range(n_seq)))
        assert len(drafts) == -(-long // step)
        for b in (3, 5, 0, 1, 22, 39):
            _, alone = decode([b], drafts)
            assert np.array_equal(alone[0], together[b][:len(alone[0])]), b
            assert len(alone[0]) == len(together[b]), b
