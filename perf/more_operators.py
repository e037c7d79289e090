"""The steps of drawing several continuations of one text, as a user's program calls them one by one: tokens drawn from truncated
distributions, scores truncated for the acceptance of drafted blocks, sequences of an 8-bit cache copied (forked, admitted from another cache, moved),
and attention of continuations over the cache of the text that they share and their own.

Truncation: w = exp((x - max x) / T).  In order of falling score (equal ones by rising index) the first top_k stay; of them the least number whose
weights sum to top_p of theirs; of them those with w >= min_p.  The drawn token is the least t whose weights up to it exceed u of all that stay.

A cache belongs to a set of sequences and heads.  Token p of a sequence lies in block p // 32; a block has one scale per head for its
keys and one for its values.  A row at position t of its sequence reads its own block in bf16 (tokens up to t) and every earlier one in 8 bits; a closed cache and the
part of a text that continuations share are read in 8 bits throughout.

Model widths and block sizes are those of `ad_inputs` (8 or 16 heads of width 64, blocks of up to 25 drafted tokens, a vocabulary of
32,000); the longer caches, the shared heads and the larger vocabulary are generic.
"""
import math

import torch

own = False

BLOCK = 32           # tokens that share a scale
E4M3_MOST = 448.0    # largest value of the 8-bit floating type
PIECE = 512          # rows that a long text is taken in by


def _sample(name, rows, vocab, scores="fp32", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, spread=2.5):
    c = dict(op="sample", rows=rows, vocab=vocab, scores=scores, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, mixed=mixed, spread=spread)
    return c if name is None else dict(c, name=name)


def _truncate(name, batch, rows_lo, rows_hi, vocab, scores="fp32", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, spread=2.5):
    c = dict(op="truncate", batch=batch, rows_lo=rows_lo, rows_hi=rows_hi, vocab=vocab, scores=scores, temperature=temperature, top_k=top_k, top_p=top_p,
             min_p=min_p, mixed=mixed, spread=spread)
    return c if name is None else dict(c, name=name)


def _copy(name, kind, texts, copies, heads, width, len_lo, len_hi, fmt="e4m3"):
    c = dict(op="copy", kind=kind, texts=texts, copies=copies, heads=heads, width=width, len_lo=len_lo, len_hi=len_hi, fmt=fmt)
    return c if name is None else dict(c, name=name)


def _shared(name, texts, each_lo, each_hi, heads, group, width, text_lo, text_hi, len_lo, len_hi, rows_lo, rows_hi, fmt="e4m3", closed=False):
    c = dict(op="shared", texts=texts, each_lo=each_lo, each_hi=each_hi, heads=heads, group=group, width=width, text_lo=text_lo, text_hi=text_hi, len_lo=len_lo,
             len_hi=len_hi, rows_lo=rows_lo, rows_hi=rows_hi, fmt=fmt, closed=closed)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # The next token of one sentence: latency.
        _sample("sample_b1_top_p", 1, 32000, temperature=0.8, top_p=0.95, spread=4.0),
        # The next tokens of 32 sentences, scores in bf16.
        _sample("sample_b32_top_k", 32, 32000, scores="bf16", temperature=0.9, top_k=50, top_p=0.9),
        # A large serving batch over a vocabulary of odd size, each request with settings of its own.
        _sample("sample_b256_mixed", 256, 100003, temperature=1.0, mixed=True, spread=3.0),
        # A sentence's drafted block before its sampled acceptance.
        _truncate("truncate_b1", 1, 8, 8, 32000, temperature=0.8, top_p=0.9, spread=4.0),
        # A batch's ragged drafted blocks, each sentence with settings of its own.
        _truncate("truncate_blocks_b32", 32, 1, 25, 32000, mixed=True),
        # One text's cache taken over by three more continuations, in the same cache: latency.
        _copy("copy_fork_b1", "fork", 1, 3, 8, 64, 301, 301),
        # Sixteen long texts, worked through in a cache of their own, admitted to the serving cache.
        _copy("copy_admit_b16_i8", "admit", 16, 1, 16, 64, 500, 8000, fmt="i8"),
        # Half of a batch's sequences ended: the last ones move to the free places.
        _copy("copy_move_b32", "move", 32, 1, 8, 128, 100, 4000),
        # Four continuations of a source-long text, one token each: latency.
        _shared("shared_token_b4", 1, 4, 4, 8, 1, 64, 512, 512, 20, 60, 1, 1),
        # Four long texts with up to 16 continuations each, drafted blocks, closed text caches of any length.
        _shared("shared_blocks_b4x16_i8", 4, 4, 16, 16, 1, 64, 2000, 8000, 1, 500, 1, 25, fmt="i8", closed=True),
        # Two very long texts, 32 continuations each, one token each, four query heads to a key head.
        _shared("shared_token_b2x32_heads", 2, 32, 32, 8, 4, 128, 16000, 32000, 100, 1000, 1, 1),
        # Many continuations of one text with drafted blocks: the products bound it.
        _shared("shared_blocks_b1x96", 1, 96, 96, 16, 1, 64, 8192, 8192, 1, 600, 8, 8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    return sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))


def draw(rng):
    kind = rng.choice(("sample", "sample", "truncate", "copy", "shared", "shared"))
    fmt = rng.choice(("e4m3", "i8"))
    heads, width = rng.choice(((8, 64), (16, 64), (4, 32), (4, 128), (3, 64)))
    if kind in ("sample", "truncate"):
        cut = dict(scores=rng.choice(("fp32", "bf16")), temperature=rng.choice((0.3, 0.7, 1.0, 1.5)), top_k=rng.choice((0, 0, 1, 40, _log_int(rng, 2, 3000))),
                   top_p=rng.choice((1.0, 0.5, 0.9, 0.99)), min_p=rng.choice((0.0, 0.0, 0.02, 0.3)), mixed=rng.random() < 0.3, spread=rng.choice((1.0, 2.5, 4.0)))
        vocab = rng.choice((2000, 32000, _log_int(rng, 100, 100003)))
        if kind == "sample":
            return _sample(None, _log_int(rng, 1, 256), vocab, **cut)
        return _truncate(None, _log_int(rng, 1, 32), *_span(rng, 1, 25), min(vocab, 32000), **cut)
    if kind == "copy":
        return _copy(None, rng.choice(("fork", "admit", "move")), _log_int(rng, 1, 16), rng.randint(1, 2), heads, width, *_span(rng, 1, 2000), fmt=fmt)
    group = rng.choice((1, 1, 2, 4))
    each = _span(rng, 1, 24 if group == 1 else 8)
    rows = _span(rng, 1, 4 if group > 1 else 8 if each[1] > 8 else 25)
    return _shared(None, rng.randint(1, 4), *each, heads, group, width, *_span(rng, 32, 6000), *_span(rng, 1, 600), *rows, fmt=fmt, closed=rng.choice((False, True)))


def _spread(lo, hi, n, seed):
    """n whole numbers spread evenly over [lo, hi], in an order made from the seed."""
    at = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
    return [int(round(lo + (hi - lo) * (i + 0.5) / n)) if hi > lo else lo for i in at]


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


# ---- inputs ------------------------------------------------------------------------------------------------------------------------
def _scores(c, seed):
    """Scores of all rows as an output projection gives them, with a few tokens that stand out, and each sequence's settings (None: not used)."""
    gen = _generator(seed)
    counts = [1] * c["rows"] if c["op"] == "sample" else _spread(c["rows_lo"], c["rows_hi"], c["batch"], seed + 2)
    n, vocab, batch = sum(counts), c["vocab"], len(counts)
    logits = c["spread"] * torch.randn((n, vocab), generator=gen, device="cuda")
    some, more = torch.randint(0, vocab, (4, n, 1), generator=gen, device="cuda"), 3 * c["spread"] * torch.rand((4, n, 1), generator=gen, device="cuda")
    for at, by in zip(some, more):
        logits.scatter_(1, at, logits.gather(1, at) + by)
    logits = logits.to({"bf16": torch.bfloat16, "fp32": torch.float32}[c["scores"]])
    if c["mixed"]:
        pick = lambda values, dtype: torch.tensor(values, dtype=dtype, device="cuda")[torch.randint(0, len(values), (batch,), generator=gen, device="cuda")]  # noqa: E731
        cut = dict(temperature=pick((0.5, 0.8, 1.0, 1.2), torch.float32), top_k=pick((0, 1, 20, 50, 1000), torch.int32),
                   top_p=pick((1.0, 0.95, 0.9, 0.5), torch.float32), min_p=pick((0.0, 0.0, 0.05), torch.float32))
    else:
        full = lambda value, none, dtype: None if value == none else torch.full((batch,), value, dtype=dtype, device="cuda")  # noqa: E731
        cut = dict(temperature=full(c["temperature"], 1.0, torch.float32), top_k=full(c["top_k"], 0, torch.int32), top_p=full(c["top_p"], 1.0, torch.float32),
                   min_p=full(c["min_p"], 0.0, torch.float32))
    return dict(logits=logits, cut=cut, u=torch.rand(n, generator=gen, device="cuda"), row_start=_i32(_starts(counts)), counts=counts)


def _values(gen, batch, tokens, heads, width):
    """Keys and values [batch, tokens, heads, width] bf16.  Keys differ in size between channels, as a projection's do."""
    channel = torch.exp(0.5 * torch.randn((heads, width), generator=gen, device="cuda")).to(torch.bfloat16)
    k = torch.randn((batch, tokens, heads, width), generator=gen, device="cuda", dtype=torch.bfloat16) * channel
    return k, torch.randn((batch, tokens, heads, width), generator=gen, device="cuda", dtype=torch.bfloat16)


def _copied(c, seed):
    """Which sequence becomes which: (source, place, lengths of all sources' sequences, sequences of the cache written to)."""
    texts, copies = c["texts"], c["copies"]
    lens = _spread(c["len_lo"], c["len_hi"], texts, seed + 1)
    if c["kind"] == "fork":      # every text behind itself, `copies` times
        return [i for i in range(texts) for _ in range(copies)], [texts + i for i in range(texts * copies)], lens, texts * (copies + 1)
    if c["kind"] == "admit":     # to free places of another cache
        return list(range(texts)), [2 * i + 1 for i in range(texts)], lens, 2 * texts
    if texts == 1:               # (one alone, from the second place to the first)
        return [1], [0], [1, lens[0]], 2
    half = texts // 2
    ended = torch.randperm(texts - half, generator=torch.Generator().manual_seed(seed + 3))[:half].tolist()
    return list(range(texts - half, texts)), ended, lens[:texts - half] + _spread(c["len_lo"], c["len_hi"], half, seed + 2), texts


def _texts(c, seed):
    """Everything an attention over shared texts is about: the texts' and the continuations' tokens, the queries, lengths and tables."""
    gen = _generator(seed)
    each = _spread(c["each_lo"], c["each_hi"], c["texts"], seed + 1)
    batch = sum(each)
    whole = 1 if c["closed"] else BLOCK
    text = [max(whole, n // whole * whole) for n in _spread(c["text_lo"], c["text_hi"], c["texts"], seed + 2)]
    lens, rows = _spread(c["len_lo"], c["len_hi"], batch, seed + 3), _spread(c["rows_lo"], c["rows_hi"], batch, seed + 4)
    shared = _values(gen, c["texts"], max(text), c["heads"], c["width"])
    mine = _values(gen, batch, max(n + r for n, r in zip(lens, rows)), c["heads"], c["width"])
    q = torch.randn((sum(rows), c["heads"] * c["group"], c["width"]), generator=gen, device="cuda", dtype=torch.bfloat16)
    return shared, mine, q, each, text, lens, rows


def _pick(t, lens, rows):
    """The packed rows [sum(rows), ..] of t [batch, tokens, ..] at tokens lens[b] .. lens[b] + rows[b] - 1."""
    return torch.cat([t[b, n:n + r] for b, (n, r) in enumerate(zip(lens, rows)) if r])


def _fill(cache, k, v, lens, piece):
    """Appends tokens [0, lens[b]) of k and v; long ones are taken in piece by piece."""
    for at in range(0, max(lens), piece):
        part, begin = [max(0, min(n - at, piece)) for n in lens], [min(at, n) for n in lens]
        cache.append(_pick(k, begin, part), _pick(v, begin, part), _i32(_starts(part)), _i32(begin))


def prepare(case, seed):
    c = case
    if c["op"] in ("sample", "truncate"):
        s = _scores(c, seed)
        return dict(s, case=dict(c), most_rows=max(s.pop("counts")))
    if c["op"] == "copy":
        source, place, lens, places = _copied(c, seed)
        k, v = _values(_generator(seed), len(lens), max(lens), c["heads"], c["width"])
        got = [lens[i] for i in source]
        back = [0] * places
        for i, n in zip(place, got):
            back[i] = n
        s = dict(case=dict(c), source=_i32(source), place=_i32(place), end=_i32(got), back_start=_i32(_starts(back)), begin=_i32([0] * places), after=_i32(back),
                 back=sum(back), most=max(got))
        if own:
            import paper_2205_10350_amd as ad
            piece = min(PIECE, max(lens))
            make = lambda n: ad.Kv8Cache(n, c["heads"], c["width"], capacity=max(lens), k_max=piece, format=c["fmt"])  # noqa: E731
            s["cache"] = make(places)
            s["origin"] = make(len(lens)) if c["kind"] == "admit" else None
            _fill(s["origin"] or s["cache"], k, v, lens + [0] * (0 if s["origin"] else places - len(lens)), piece)
            return s
        s["held"] = [_held(t, lens, c["fmt"]) for t in (k, v)]
        s["room"] = [tuple(torch.zeros((places, *t.shape[1:]), dtype=t.dtype, device="cuda") for t in h) for h in s["held"]]
        return s
    shared, mine, q, each, text, lens, rows = _texts(c, seed)
    s = dict(case=dict(c), q=q, length=_i32(lens), row_start=_i32(_starts(rows)), seq_start=_i32(_starts(each)), text=_i32(text), most_rows=max(rows),
             most_keys=max(n + r for n, r in zip(lens, rows)), most_text=max(text))
    first = _starts(each)
    s["most_text_rows"] = max(sum(rows[a:b]) for a, b in zip(first, first[1:]))
    if own:
        import paper_2205_10350_amd as ad
        piece = min(PIECE, max(text))
        s["shared"] = ad.Kv8Cache(len(text), c["heads"], c["width"], capacity=max(text), k_max=piece, format=c["fmt"], closed=c["closed"])
        _fill(s["shared"], *shared, text, max(text) if c["closed"] else piece)
        s["cache"] = ad.Kv8Cache(len(lens), c["heads"], c["width"], capacity=s["most_keys"], k_max=max(max(rows), min(max(lens), PIECE)), format=c["fmt"])
        _fill(s["cache"], *mine, lens, min(max(lens), PIECE))
        s["cache"].append(*(_pick(t, lens, rows) for t in mine), s["row_start"], s["length"])
        return s
    # The same as tensors: 8-bit blocks with their scales, and the bf16 tokens from each sequence's incomplete block on.
    live = torch.arange(s["most_text"], device="cuda")[None, :] < s["text"][:, None]
    s["held_text"] = [_quantised(_blocks(torch.where(live[:, :, None, None], t, 0)), c["fmt"]) for t in shared]
    s["held"] = [_quantised(_blocks(t), c["fmt"]) for t in mine]
    base = [n // BLOCK * BLOCK for n in lens]
    wide = max(n + r - f for n, r, f in zip(lens, rows, base))
    s["recent"] = [torch.stack([torch.nn.functional.pad(t[b, f:f + wide], (0, 0, 0, 0, 0, wide - t[b, f:f + wide].shape[0])) for b, f in enumerate(base)])
                   for t in mine]
    return s


# ---- the plain form ----------------------------------------------------------------------------------------------------------------
def _blocks(t):
    """[batch, tokens, heads, width] -> [batch, heads, blocks, 32, width], the last block filled up with zeros."""
    t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, -t.shape[1] % BLOCK))
    return t.view(t.shape[0], -1, BLOCK, t.shape[2], t.shape[3]).permute(0, 3, 1, 2, 4)


def _quantised(x, fmt):
    """8-bit values and fp32 scales [.., 1, 1] of blocks [.., 32, width]."""
    most = x.abs().amax((-2, -1), keepdim=True).float()
    if fmt == "e4m3":
        m, e = torch.frexp(most)                                   # most = m 2^e: the least power of two that brings it to 448 = 0.875 * 2^9
        e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
        e = torch.where(most == 0, 0, e)
        scale = torch.ldexp(torch.ones_like(most), e)
        return (x.float() * torch.ldexp(torch.ones_like(most), -e)).to(torch.float8_e4m3fn), scale
    # (in 64 bits: halves between two steps have to be seen as halves)
    held = torch.round(x.double() * 127 / torch.where(most == 0, 1, most).double()).to(torch.int8)
    return held, torch.where(most == 0, 1, most / 127)


def _held(t, lens, fmt):
    """A cache's tensors: 8-bit blocks, their scales, and the incomplete block's tokens [batch, 32, heads, width] in bf16."""
    q, scale = _quantised(_blocks(t), fmt)
    recent = torch.stack([torch.nn.functional.pad(t[b, n // BLOCK * BLOCK:n], (0, 0, 0, 0, 0, BLOCK - n % BLOCK)) for b, n in enumerate(lens)])
    return q.contiguous().view(torch.int8), scale, recent


def _plain_weights(s):
    """Weights of all rows' tokens in 64 bits (0: cut off), and (x - max x) / T."""
    # in 64 bits: a drawn number or a sum may lie next to the border between two tokens
    x = s["logits"].double()
    start, cut = s["row_start"].long(), s["cut"]
    which = torch.repeat_interleave(torch.arange(start.shape[0] - 1, device="cuda"), start[1:] - start[:-1], output_size=x.shape[0])
    z = x - x.amax(-1, keepdim=True)
    if cut["temperature"] is not None:
        z = z / cut["temperature"].double()[which, None]
    w = torch.exp(z)
    if cut["top_k"] is None and cut["top_p"] is None:
        keep = torch.ones_like(w, dtype=torch.bool)
    else:
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices
        sorted_w = w.gather(1, order)
        rank = torch.arange(w.shape[1], device="cuda")[None, :]
        keep = torch.ones_like(w, dtype=torch.bool)
        if cut["top_k"] is not None:
            k = cut["top_k"].long()[which, None]
            keep = (k <= 0) | (rank < k)
            sorted_w = torch.where(keep, sorted_w, 0)
        if cut["top_p"] is not None:
            p = cut["top_p"].double()[which, None]
            sums = sorted_w.cumsum(-1)
            before = torch.nn.functional.pad(sums[:, :-1], (1, 0))
            keep = keep & ((p >= 1) | (before < p * sums[:, -1:]) | (rank == 0))
        keep = torch.zeros_like(keep).scatter_(1, order, keep)
    if cut["min_p"] is not None:
        keep = keep & (w >= cut["min_p"].double()[which, None])
    return torch.where(keep, w, 0), keep, z


def _plain_sample(s):
    w, _, z = _plain_weights(s)
    sums = w.cumsum(-1)
    token = (sums <= s["u"].double()[:, None] * sums[:, -1:]).sum(-1).clamp(max=w.shape[1] - 1)
    log_prob = z.gather(1, token[:, None])[:, 0] - torch.log(sums[:, -1])
    return {"tokens": token.to(torch.int32), "log_probs": log_prob.float()}


def _plain_truncate(s):
    return torch.where(_plain_weights(s)[1], s["logits"], -math.inf)


def _plain_copy(s):
    c = s["case"]
    source, place = s["source"].long(), s["place"].long()
    start, after = s["back_start"].long(), s["after"].long()
    which = torch.repeat_interleave(torch.arange(after.shape[0], device="cuda"), after, output_size=s["back"])
    at = torch.arange(s["back"], device="cuda") - start[which]
    out = {}
    for name, held, room in zip("kv", s["held"], s["room"]):
        for t, r in zip(held, room):
            r[place] = t[source]
        q, scale, recent = room
        blk = at // BLOCK
        values = q.view(torch.float8_e4m3fn if c["fmt"] == "e4m3" else torch.int8)
        # (row by row: block and token of each, all heads)
        read = values.view(torch.int8).permute(0, 2, 3, 1, 4)[which, blk, at % BLOCK].view(values.dtype).float() * scale[:, :, :, 0, 0].permute(0, 2, 1)[which, blk][:, :, None]
        whole = (blk + 1) * BLOCK <= after[which]
        out[name] = torch.where(whole[:, None, None], read, recent[which, at % BLOCK].float()).to(torch.bfloat16)
    return out


def _part(q, k, v, seen):
    """Attention's maximum, sum and product of scaled queries [.., rows, width] over keys [.., keys, width], of what each row sees."""
    x = torch.where(seen, q @ k.transpose(-1, -2), -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0, top))
    return top, w.sum(-1, keepdim=True), w @ v


def _plain_shared(s):
    c = s["case"]
    heads, group, width = c["heads"], c["group"], c["width"]
    start, seq_start, length, text = (s[n].long() for n in ("row_start", "seq_start", "length", "text"))
    total = s["q"].shape[0]

    def padded(first, n):            # packed rows first[i] .. as [i, heads, group * n, width], and a table to take results back by
        at = (first[:-1, None] + torch.arange(n, device="cuda")).clamp(max=total - 1)
        q = s["q"][at].float().view(at.shape[0], n, heads, group, width).permute(0, 2, 3, 1, 4).reshape(at.shape[0], heads, group * n, width)
        which = torch.repeat_interleave(torch.arange(at.shape[0], device="cuda"), first[1:] - first[:-1], output_size=total)
        return q / math.sqrt(width), which, torch.arange(total, device="cuda") - first[which]

    def packed(t, which, place, n):
        return t.view(t.shape[0], heads, group, n, -1).permute(0, 3, 1, 2, 4)[which, place].reshape(total, heads * group, -1)

    def held(pair):
        return [(t.float() * sc).reshape(t.shape[0], heads, -1, width) for t, sc in pair]

    q, which, place = padded(start[seq_start], s["most_text_rows"])
    k, v = held(s["held_text"])
    seen = torch.arange(k.shape[2], device="cuda")[None, :] < text[:, None]
    parts = [[packed(t, which, place, s["most_text_rows"]) for t in _part(q, k, v, seen[:, None, None, :])]]
    n = s["most_rows"]
    q, which, place = padded(start, n)
    k, v = held(s["held"])
    t = length[:, None] + torch.arange(n, device="cuda")                            # a row's position
    seen = torch.arange(k.shape[2], device="cuda")[None, None, :] < (t // BLOCK * BLOCK)[:, :, None]
    own_k, own_v = (r.float().permute(0, 2, 1, 3) for r in s["recent"])
    p = (length // BLOCK * BLOCK)[:, None] + torch.arange(own_k.shape[2], device="cuda")
    own_seen = (p[:, None, :] // BLOCK == t[:, :, None] // BLOCK) & (p[:, None, :] <= t[:, :, None])
    k, v, seen = torch.cat((k, own_k), 2), torch.cat((v, own_v), 2), torch.cat((seen, own_seen), 2)
    seen = seen[:, None, None].expand(-1, 1, group, n, -1).reshape(seen.shape[0], 1, group * n, -1)
    parts.append([packed(t, which, place, n) for t in _part(q, k, v, seen)])
    (m0, l0, o0), (m1, l1, o1) = parts
    top = torch.maximum(m0, m1)
    f0, f1 = torch.exp(m0 - top), torch.exp(m1 - top)
    return ((o0 * f0 + o1 * f1) / (l0 * f0 + l1 * f1)).to(torch.bfloat16)


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"sample": _plain_sample, "truncate": _plain_truncate, "copy": _plain_copy, "shared": _plain_shared}[op](s)
    import paper_2205_10350_amd as ad

    if op == "sample":
        tokens, log_probs = ad.sample_tokens(s["logits"], s["u"], log_probs=True, **s["cut"])
        return {"tokens": tokens, "log_probs": log_probs}
    if op == "truncate":
        return ad.truncate_scores(s["logits"], row_start=s["row_start"], **s["cut"])
    if op == "copy":
        s["cache"].copy(s["source"], s["place"], s["end"], origin=s["origin"], max_tokens=s["most"])
        k, v = s["cache"].read(s["back_start"], s["begin"], s["after"], rows=s["back"], max_rows=s["most"])
        return {"k": k, "v": v}
    return s["cache"].attend_shared(s["q"], s["row_start"], s["length"], s["shared"], s["seq_start"], s["text"], max_rows=s["most_rows"], max_keys=s["most_keys"],
                                    max_shared_rows=s["most_text_rows"], max_shared_keys=s["most_text"])


def work(case):
    """What has to cross memory once, at the mean lengths: 8 bits a value of a key or value that is read or copied, 16 of one that is given back."""
    c = case
    if c["op"] in ("sample", "truncate"):
        rows = c["rows"] if c["op"] == "sample" else c["batch"] * (c["rows_lo"] + c["rows_hi"]) / 2
        size = 4 if c["scores"] == "fp32" else 2
        return {"bytes": rows * (c["vocab"] * size * (1 if c["op"] == "sample" else 2) + 12), "flops": 4 * rows * c["vocab"]}
    values = 2 * c["heads"] * c["width"]
    if c["op"] == "copy":
        n = {"fork": c["texts"] * c["copies"], "admit": c["texts"], "move": max(c["texts"] // 2, 1)}[c["kind"]] * (c["len_lo"] + c["len_hi"]) / 2
        return {"bytes": n * values * 4, "flops": n * values}
    batch = c["texts"] * (c["each_lo"] + c["each_hi"]) / 2
    text, mine, each = (c["text_lo"] + c["text_hi"]) / 2, (c["len_lo"] + c["len_hi"]) / 2, (c["rows_lo"] + c["rows_hi"]) / 2
    q = c["heads"] * c["group"] * c["width"]
    return {"bytes": (c["texts"] * text + batch * mine) * values * (1 + 4 / (BLOCK * c["width"])) + 2 * batch * each * values + 4 * batch * each * q,
            "flops": 4 * batch * each * q * (text + mine + each / 2)}


# ---- from the definitions, in 64 bits -------------------------------------------------------------------------------------------------
def _exact_held(x, fmt):
    """What a complete block [.., 32, width] stands for: float64 in, float64 out."""
    most = x.abs().amax((-2, -1), keepdim=True)
    if fmt == "i8":
        step = torch.where(most > 0, most, 127.0) / 127
        return torch.round(torch.where(most > 0, x * 127 / torch.where(most > 0, most, 1.0), 0.0)) * step
    _, e = torch.frexp(most / E4M3_MOST)
    unit = torch.exp2(torch.where(most / E4M3_MOST == torch.exp2((e - 1).double()), e - 1, e).clamp(min=-126).double())
    y = torch.where(most > 0, x / unit, 0.0)
    # a value of size [2^a, 2^(a+1)) has steps of 2^(a-3); below 2^-6 all steps are 2^-9
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * unit


def _exact_tokens(t, tokens, fmt, closed):
    """t [tokens, heads, width] as the row behind the last token reads it: complete blocks in 8 bits (closed: all)."""
    full = -(-tokens // BLOCK) * BLOCK if closed else tokens // BLOCK * BLOCK
    x = torch.nn.functional.pad(t[:tokens].double(), (0, 0, 0, 0, 0, max(0, full - tokens)))
    if full:
        blocks = x[:full].view(-1, BLOCK, *x.shape[1:]).transpose(1, 2)
        x = torch.cat((_exact_held(blocks, fmt).transpose(1, 2).reshape(full, *x.shape[1:]), x[full:]))
    return x[:tokens]


def _exact_kept(x, seq, cut):
    """Tokens of one row of scores (float64) that stay, and the probabilities among all."""
    at = lambda name, none: none if cut[name] is None else cut[name][seq].item()  # noqa: E731
    p = torch.softmax(x / at("temperature", 1.0), 0)
    k, top_p, min_p = at("top_k", 0), at("top_p", 1.0), at("min_p", 0.0)
    by = torch.argsort(-x, stable=True)
    if 0 < k < x.shape[0]:
        by = by[:k]
    if top_p < 1:
        sums = torch.cumsum(p[by], 0)
        by = by[:int(torch.searchsorted(sums, top_p * sums[-1:])) + 1]
    kept = torch.zeros_like(x, dtype=torch.bool)
    kept[by] = True
    return kept & (p / p.max() >= min_p), p


def exact(case, seed):
    c = case
    if c["op"] in ("sample", "truncate"):
        return _exact_scores(c, seed)
    if c["op"] == "copy":
        source, place, lens, places = _copied(c, seed)
        k, v = _values(_generator(seed), len(lens), max(lens), c["heads"], c["width"])
        return {name: torch.cat([_exact_tokens(t[i], lens[i], c["fmt"], False) for _, i in sorted(zip(place, source))]) for name, t in (("k", k), ("v", v))}
    shared, mine, q, each, text, lens, rows = _texts(c, seed)
    starts, parts, b = _starts(rows), [], 0
    for g, count in enumerate(each):
        front = [_exact_tokens(t[g], text[g], c["fmt"], True).repeat_interleave(c["group"], 1).transpose(0, 1) for t in shared]
        for b in range(b, b + count):
            n, r = lens[b], rows[b]
            raw = [torch.cat((f, t[b, :n + r].double().repeat_interleave(c["group"], 1).transpose(0, 1)), 1) for t, f in zip(mine, front)]
            held = [torch.cat((f, _exact_tokens(t[b], n + r, c["fmt"], False).repeat_interleave(c["group"], 1).transpose(0, 1)), 1) for t, f in zip(mine, front)]
            t = torch.arange(n, n + r, device="cuda")[:, None]
            key = torch.arange(-text[g], n + r, device="cuda")[None, :]
            qq = q[starts[b]:starts[b] + r].double().transpose(0, 1) / math.sqrt(c["width"])
            near = (key >= 0) & (key // BLOCK == t // BLOCK)
            x = torch.where(near, qq @ raw[0].transpose(1, 2), qq @ held[0].transpose(1, 2))
            w = torch.softmax(torch.where(key <= t, x, -math.inf), -1)
            parts.append((torch.where(near, 0.0, w) @ held[1] + torch.where(near, w, 0.0) @ raw[1]).transpose(0, 1))
        b += 1
    return torch.cat(parts)


def _exact_scores(c, seed):
    s = _scores(c, seed)
    at, u = s["row_start"].tolist(), s["u"].tolist()
    tokens, log_probs, scores = [], [], []
    for seq in range(len(at) - 1):
        for r in range(at[seq], at[seq + 1]):
            x = s["logits"][r].double()
            kept, p = _exact_kept(x, seq, s["cut"])
            if c["op"] == "truncate":
                scores.append(torch.where(kept, x, -math.inf))
                continue
            there = kept.nonzero()[:, 0]
            sums = torch.cumsum(p[there], 0)
            got = int(torch.searchsorted(sums, u[r] * sums[-1:], right=True))
            tokens.append(int(there[got]))
            log_probs.append(torch.log(p[there[got]] / sums[-1]))
    if c["op"] == "truncate":
        return torch.stack(scores)
    return {"tokens": _i32(tokens), "log_probs": torch.stack(log_probs)}
