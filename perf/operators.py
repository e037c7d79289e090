"""The steps of a sampled block verification over key/value caches in 8 bits, as a user's program calls them one by one:
rows written to a cache and read back, attention of a block of rows over the cache, and the acceptance of drafted tokens.

A cache belongs to a set of sequences and heads.  Token p of a sequence lies in block p // 32; a block has one scale per head for its
keys and one for its values.  A row at position t reads its own block in bf16 (tokens up to t) and every earlier one in 8 bits, so that
what a row reads does not depend on how the tokens came in.  A closed cache (an encoder's memory) is written at once and read in 8 bits throughout.

Model widths and block sizes are those of `ad_inputs` (8 or 16 heads of width 64, blocks of up to 25 drafted tokens, a vocabulary of
32,000, sources of up to 512 tokens); the longer caches, the shared heads and the larger vocabulary are generic.
"""
import math

import torch

own = False

BLOCK = 32           # tokens that share a scale
E4M3_MOST = 448.0    # largest value of the 8-bit floating type


def _write(name, batch, heads, width, len_lo, len_hi, rows_lo, rows_hi, fmt="e4m3", values="bf16", closed=False):
    c = dict(op="write", batch=batch, heads=heads, width=width, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo, rows_hi=rows_hi,
             fmt=fmt, values=values, closed=closed)
    return c if name is None else dict(c, name=name)


def _attend(name, batch, heads, shared, width, len_lo, len_hi, rows_lo, rows_hi, fmt="e4m3", closed=False):
    c = dict(op="attend", batch=batch, heads=heads, shared=shared, width=width, len_lo=len_lo, len_hi=len_hi, rows_lo=rows_lo,
             rows_hi=rows_hi, fmt=fmt, closed=closed)
    return c if name is None else dict(c, name=name)


def _accept(name, batch, rows_lo, rows_hi, vocab, scores="fp32", drafter=False, temperature=1.0):
    c = dict(op="accept", batch=batch, rows_lo=rows_lo, rows_hi=rows_hi, vocab=vocab, scores=scores, drafter=drafter, temperature=temperature)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # One token of one sentence appended by an autoregressive step of the base model: latency.
        _write("write_token_b1", 1, 8, 64, 40, 40, 1, 1),
        # A batch's drafted blocks, ragged, behind outputs of all lengths.
        _write("write_blocks_b32_i8", 32, 8, 64, 100, 4000, 1, 25, fmt="i8", values="fp32"),
        # Long prompts taken in at once by the wide model.
        _write("write_prompts_b8", 8, 16, 64, 0, 0, 1000, 2048),
        # One decoder row over a short output (base model): latency.
        _attend("attend_token_b1", 1, 8, 1, 64, 40, 40, 1, 1),
        # A drafted block over one long output.
        _attend("attend_block_b1_long", 1, 16, 1, 64, 8191, 8191, 25, 25),
        # Cross-attention of drafted blocks to the memories of eight long documents.
        _attend("attend_memory_b8", 8, 16, 1, 64, 301, 512, 25, 25, closed=True),
        # A serving batch: ragged lengths from one token on, ragged blocks.
        _attend("attend_blocks_b32_i8", 32, 16, 1, 64, 1, 8192, 1, 25, fmt="i8"),
        # One token each over very long caches, four query heads to a key head of width 128.
        _attend("attend_token_b8_shared", 8, 8, 4, 128, 16000, 32000, 1, 1),
        # A piece of a long prompt over what came before it: the products bound it.
        _attend("attend_prompt_b2", 2, 16, 1, 64, 4000, 8000, 512, 512),
        # One sentence's drafted block from a drafter that gives tokens only (the block drafter, an input as guide).
        _accept("accept_b1", 1, 8, 8, 32000),
        # A batch's drafted blocks from a drafter that gives its probabilities.
        _accept("accept_probs_b32", 32, 1, 25, 32000, drafter=True, temperature=0.8),
        # Many short blocks over a large vocabulary of odd size, scores in bf16.
        _accept("accept_b64_bf16", 64, 3, 8, 100003, scores="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    return sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))


def draw(rng):
    kind = rng.choice(("write", "prompt", "attend", "attend", "shared", "memory", "piece", "accept", "probs"))
    fmt = rng.choice(("e4m3", "i8"))
    batch = _log_int(rng, 1, 32)
    heads, width = rng.choice(((8, 64), (16, 64), (4, 32), (4, 128), (3, 64)))
    if kind == "write":
        return _write(None, batch, heads, width, *_span(rng, 1, 4000), *_span(rng, 1, 72), fmt=fmt, values=rng.choice(("bf16", "fp32")))
    if kind == "prompt":
        return _write(None, _log_int(rng, 1, 8), heads, width, 0, 0, *_span(rng, 20, 2048), fmt=fmt, closed=rng.choice((False, True)))
    if kind == "attend":
        return _attend(None, batch, heads, 1, width, *_span(rng, 1, 8192), *_span(rng, 1, 72), fmt=fmt)
    if kind == "shared":
        return _attend(None, _log_int(rng, 1, 8), rng.randint(1, 8), rng.choice((2, 3, 4, 8)), 128, *_span(rng, 100, 32000), *_span(rng, 1, 8), fmt=fmt)
    if kind == "memory":
        return _attend(None, batch, heads, 1, width, *_span(rng, 1, 2000), *_span(rng, 1, 72), fmt=fmt, closed=True)
    if kind == "piece":
        return _attend(None, rng.randint(1, 2), heads, 1, width, *_span(rng, 1, 8000), *_span(rng, 64, 512), fmt=fmt)
    vocab = rng.choice((2000, 32000, _log_int(rng, 100, 100003)))
    if kind == "probs":
        return _accept(None, batch, *_span(rng, 1, 25), min(vocab, 32000), drafter=True, temperature=rng.choice((0.5, 0.8, 1.0, 1.3)))
    return _accept(None, batch, *_span(rng, 1, 8), vocab, scores=rng.choice(("fp32", "bf16")), temperature=rng.choice((0.7, 1.0)))


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


def _type(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def _counts(c, seed):
    lens = [0] * c["batch"] if c["op"] == "accept" else _spread(c["len_lo"], c["len_hi"], c["batch"], seed + 1)
    return lens, _spread(c["rows_lo"], c["rows_hi"], c["batch"], seed + 2)


def _tokens(c, seed):
    """Keys and values of all tokens of every sequence, [batch, tokens, heads, width] bf16 (those in the cache and those being written), and
    the queries [rows, query heads, width].  Keys differ in size between channels, as a projection's do; scores come out a few units wide."""
    lens, rows = _counts(c, seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    most = max(n if c["closed"] and c["op"] == "attend" else n + r for n, r in zip(lens, rows))
    shape = (c["batch"], most, c["heads"], c["width"])
    channel = torch.exp(0.5 * torch.randn((c["heads"], c["width"]), generator=gen, device="cuda"))
    k = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16) * channel.to(torch.bfloat16)
    v = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    q = None
    if c["op"] == "attend":
        q = torch.randn((sum(rows), c["heads"] * c["shared"], c["width"]), generator=gen, device="cuda", dtype=torch.bfloat16)
    return k, v, q, lens, rows


def _pick(t, lens, rows):
    """The packed rows [sum(rows), ..] of t [batch, tokens, ..] at tokens lens[b] .. lens[b] + rows[b] - 1."""
    return torch.cat([t[b, n:n + r] for b, (n, r) in enumerate(zip(lens, rows))])


def _scores(c, seed):
    """Scores of all rows as an output projection gives them, the drafter's tokens and probabilities, and the random numbers."""
    _, rows = _counts(c, seed)
    gen = torch.Generator("cuda").manual_seed(seed)
    n, vocab = sum(rows), c["vocab"]
    logits = (2.5 * torch.randn((n, vocab), generator=gen, device="cuda")).to(_type(c["scores"]))
    probs = torch.softmax((logits.float() + 0.7 * torch.randn((n, vocab), generator=gen, device="cuda")) / c["temperature"], -1)
    draft = torch.multinomial(probs, 1, generator=gen).view(n).to(torch.int32)
    if not c["drafter"]:
        draft = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.8, logits.argmax(-1).to(torch.int32), draft)
        # such drafters' tokens stand often: the target is sure of most of them
        logits.scatter_add_(1, logits.argmax(-1, keepdim=True), torch.full((n, 1), 8.0, device="cuda", dtype=logits.dtype))
    return dict(logits=logits, draft=draft, probs=probs if c["drafter"] else None,
                accept_u=torch.rand(n, generator=gen, device="cuda"), pick_u=torch.rand(c["batch"], generator=gen, device="cuda"),
                temperature=torch.full((c["batch"],), c["temperature"], device="cuda"), row_start=_i32(_starts(rows)), most_rows=max(rows))


def _cache(c, k, v, lens, rows):
    """A cache of the framework holding tokens [0, lens[b]), with room for the rows to come; long ones are taken in piece by piece."""
    import paper_2205_10350_amd as ad

    capacity = max(n + r for n, r in zip(lens, rows))
    piece = max(lens) if c["closed"] and max(lens) else min(max(512, max(rows)), capacity)
    if c["closed"] and c["op"] == "write":
        piece = capacity
    cache = ad.Kv8Cache(c["batch"], c["heads"], c["width"], capacity=capacity, k_max=piece, format=c["fmt"], closed=c["closed"])
    for at in range(0, max(lens), piece):
        part = [max(0, min(n - at, piece)) for n in lens]
        begin = [min(at, n) for n in lens]
        cache.append(_pick(k, begin, part), _pick(v, begin, part), _i32(_starts(part)), _i32(begin))
    return cache


def prepare(case, seed):
    c = case
    if c["op"] == "accept":
        return dict(_scores(c, seed), case=dict(c))
    k, v, q, lens, rows = _tokens(c, seed)
    s = dict(case=dict(c), q=q, length=_i32(lens), row_start=_i32(_starts(rows)), most_rows=max(rows), most_keys=max(n + r for n, r in zip(lens, rows)))
    if c["op"] == "write":
        first = [n // BLOCK * BLOCK for n in lens]      # what is read back: the blocks that the call writes to, from their first token on
        back = [n + r - f for n, r, f in zip(lens, rows, first)]
        s.update(k=_pick(k, lens, rows), v=_pick(v, lens, rows), after=_i32([n + r for n, r in zip(lens, rows)]), begin=_i32(first),
                 back_start=_i32(_starts(back)), back=sum(back), most_back=max(back))
        if own:
            s["cache"] = _cache(c, k, v, lens, rows)
        else:                                           # the incomplete blocks' earlier tokens, which a cache keeps as they are
            keep = torch.arange(BLOCK, device="cuda")[None, :] < (s["length"] - s["begin"])[:, None]
            at = (s["begin"].long()[:, None] + torch.arange(BLOCK, device="cuda")[None, :]).clamp_(max=k.shape[1] - 1)
            s["recent"] = [torch.where(keep[:, :, None, None], t[torch.arange(c["batch"], device="cuda")[:, None], at], 0) for t in (k, v)]
        return s
    if c["closed"]:
        s["most_keys"] = max(lens)
    if own:
        s["cache"] = _cache(c, k, v, lens, [0] * len(lens) if c["closed"] else rows)
        if not c["closed"]:
            s["cache"].append(_pick(k, lens, rows), _pick(v, lens, rows), s["row_start"], s["length"])
        return s
    # The same as tensors: 8-bit blocks with their scales, and the bf16 tokens from each sequence's incomplete block on.
    if c["closed"]:
        k, v = (torch.where(torch.arange(t.shape[1], device="cuda")[None, :, None, None] < s["length"][:, None, None, None], t, 0) for t in (k, v))
    s["held"] = [_quantised(_blocks(t), c["fmt"]) for t in (k, v)]
    base = [n // BLOCK * BLOCK for n in lens]
    wide = max(n + r - f for n, r, f in zip(lens, rows, base))
    s["recent"] = [torch.stack([torch.nn.functional.pad(t[b, f:f + wide], (0, 0, 0, 0, 0, wide - t[b, f:f + wide].shape[0])) for b, f in enumerate(base)])
                   for t in (k, v)] if not c["closed"] else None
    return s


# ---- the plain form ----------------------------------------------------------------------------------------------------------
def _blocks(t):
    """[batch, tokens, heads, width] -> [batch, heads, blocks, 32, width], the last block filled up with zeros."""
    pad = -t.shape[1] % BLOCK
    t = torch.nn.functional.pad(t, (0, 0, 0, 0, 0, pad))
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


def _plain_write(s):
    c = s["case"]
    batch = c["batch"]
    begin, length, after, start = (s[n].long() for n in ("begin", "length", "after", "row_start"))
    wide = -(-(s["most_rows"] + BLOCK - 1) // BLOCK) * BLOCK
    at = torch.arange(wide, device="cuda")[None, :] + begin[:, None]                  # token of each place
    new = (at - length[:, None]).clamp(min=0) + start[:batch, None]
    back_start = s["back_start"].long()
    which = torch.repeat_interleave(torch.arange(batch, device="cuda"), back_start[1:] - back_start[:-1], output_size=s["back"])
    place = torch.arange(s["back"], device="cuda") - back_start[which]

    def values(rows, recent):
        t = rows[new.clamp(max=rows.shape[0] - 1)]
        t = torch.where((at < length[:, None])[:, :, None, None], torch.nn.functional.pad(recent, (0, 0, 0, 0, 0, wide - BLOCK)), t)
        t = torch.where((at < after[:, None])[:, :, None, None], t, 0)
        held, scale = _quantised(_blocks(t), c["fmt"])
        read = (held.float() * scale).permute(0, 2, 3, 1, 4).reshape(t.shape)
        whole = c["closed"] | ((at // BLOCK + 1) * BLOCK <= after[:, None])
        read = torch.where(whole[:, :, None, None], read, t.float())
        return read[which, place].to(_type(c["values"]))

    return {"k": values(s["k"], s["recent"][0]), "v": values(s["v"], s["recent"][1])}


def _plain_attend(s):
    c = s["case"]
    batch, heads, width, n = c["batch"], c["heads"], c["width"], s["most_rows"]
    length, start = s["length"].long(), s["row_start"].long()
    i = torch.arange(n, device="cuda")
    rows = (start[:batch, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][rows].float().view(batch, n, heads, c["shared"], width).permute(0, 2, 3, 1, 4).reshape(batch, heads, -1, width)
    (kq, ks), (vq, vs) = s["held"]
    k, v = ((t.float() * sc).view(batch, heads, -1, width) for t, sc in ((kq, ks), (vq, vs)))
    key = torch.arange(k.shape[2], device="cuda")
    if c["closed"]:
        seen = (key[None, :] < length[:, None])[:, None, :].expand(batch, n, -1)
    else:
        t = length[:, None] + i                                                         # a row's position
        seen = key[None, None, :] < (t // BLOCK * BLOCK)[:, :, None]
        own_k, own_v = (r.float().permute(0, 2, 1, 3) for r in s["recent"])
        p = (length // BLOCK * BLOCK)[:, None] + torch.arange(own_k.shape[2], device="cuda")
        own_seen = (p[:, None, :] // BLOCK == t[:, :, None] // BLOCK) & (p[:, None, :] <= t[:, :, None])
        k, v, seen = torch.cat((k, own_k), 2), torch.cat((v, own_v), 2), torch.cat((seen, own_seen), 2)
    seen = seen[:, None, None].expand(batch, 1, c["shared"], n, -1).reshape(batch, 1, c["shared"] * n, -1)
    x = torch.where(seen, (q @ k.transpose(2, 3)) / math.sqrt(width), -math.inf)
    top = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(top == -math.inf, 0, top))
    total = w.sum(-1, keepdim=True)
    o = (w @ v) / torch.where(total == 0, 1, total)
    o = o.view(batch, heads, c["shared"], n, width).permute(0, 3, 1, 2, 4).reshape(batch, n, -1, width)
    which = torch.repeat_interleave(torch.arange(batch, device="cuda"), start[1:] - start[:-1], output_size=s["q"].shape[0])
    return o[which, torch.arange(s["q"].shape[0], device="cuda") - start[which]].to(torch.bfloat16)


def _plain_accept(s):
    # in 64 bits: a drawn number may lie next to the border between two tokens
    vocab, start = s["logits"].shape[1], s["row_start"].long()
    count = start[1:] - start[:-1]
    which = torch.repeat_interleave(torch.arange(count.shape[0], device="cuda"), count, output_size=s["draft"].shape[0])
    x = s["logits"].double() / s["temperature"].double()[which, None]
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    d = s["draft"].long()[:, None]
    drafted = torch.ones_like(s["accept_u"], dtype=torch.float64) if s["probs"] is None else s["probs"].gather(1, d)[:, 0].double()
    stands = s["accept_u"].double() * drafted < p.gather(1, d)[:, 0]
    i = torch.arange(s["most_rows"], device="cuda")
    rows = (start[:-1, None] + i).clamp(max=which.shape[0] - 1)
    before = torch.where(i < count[:, None], stands[rows], False).long().cumprod(1).sum(1)       # drafted tokens that stand
    decide = (start[:-1] + before).clamp(max=which.shape[0] - 1)
    left = p[decide]
    if s["probs"] is None:
        left = left.scatter(1, d[decide], 0.0)
    else:
        left = (left - s["probs"][decide].double()).clamp(min=0)
    sums = left.cumsum(-1)
    token = (sums <= s["pick_u"].double()[:, None] * sums[:, -1:]).sum(-1).clamp(max=vocab - 1)
    token = torch.where(sums[:, -1] > 0, token, s["draft"].long()[decide])
    place = torch.arange(which.shape[0], device="cuda") - start[which]
    out = torch.where(place < before[which], s["draft"].long(), torch.where(place == before[which], token[which], -1))
    return {"accepted": torch.minimum(before + 1, count).to(torch.int32), "tokens": out.to(torch.int32)}


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"write": _plain_write, "attend": _plain_attend, "accept": _plain_accept}[op](s)
    if op == "write":
        s["cache"].append(s["k"], s["v"], s["row_start"], s["length"], max_rows=s["most_rows"])
        k, v = s["cache"].read(s["back_start"], s["begin"], s["after"], rows=s["back"], max_rows=s["most_back"], dtype=_type(s["case"]["values"]))
        return {"k": k, "v": v}
    if op == "attend":
        return s["cache"].attend(s["q"], s["row_start"], s["length"], max_rows=s["most_rows"], max_keys=s["most_keys"])
    import paper_2205_10350_amd as ad

    accepted, tokens = ad.accept_sampled(s["logits"], s["draft"], s["row_start"], s["accept_u"], s["pick_u"], temperature=s["temperature"],
                                         draft_probs=s["probs"], max_rows=s["most_rows"])
    return {"accepted": accepted, "tokens": tokens}


def work(case):
    """What has to cross memory once, at the mean lengths: 8 bits a value of a key or value that is read or finished, 16 of one that comes in."""
    c = case
    rows = c["batch"] * (c["rows_lo"] + c["rows_hi"]) / 2
    if c["op"] == "accept":
        size = 4 if c["scores"] == "fp32" else 2
        return {"bytes": rows * (c["vocab"] * size + 16) + (c["batch"] * c["vocab"] * 4 if c["drafter"] else 0), "flops": 3 * rows * c["vocab"]}
    values = 2 * c["heads"] * c["width"]
    tokens = c["batch"] * (c["len_lo"] + c["len_hi"]) / 2
    if c["op"] == "write":
        back = 2 if c["values"] == "bf16" else 4
        return {"bytes": rows * values * (2 + 1 + 1 + back), "flops": 4 * rows * values}
    keys = (c["len_lo"] + c["len_hi"]) / 2 + (0 if c["closed"] else (c["rows_lo"] + c["rows_hi"]) / 4)
    q = c["heads"] * c["shared"] * c["width"]
    return {"bytes": tokens * values * (1 + 4 / (BLOCK * c["width"])) + (0 if c["closed"] else 2 * rows * values) + 4 * rows * q,
            "flops": 4 * rows * q * keys}


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------------------------
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
    x = t[:tokens].double()
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, max(0, full - tokens)))
    if full:
        blocks = x[:full].view(-1, BLOCK, *x.shape[1:]).transpose(1, 2)
        x = torch.cat((_exact_held(blocks, fmt).transpose(1, 2).reshape(full, *x.shape[1:]), x[full:]))
    return x[:tokens]


def exact(case, seed):
    c = case
    if c["op"] == "accept":
        return _exact_accept(c, seed)
    k, v, q, lens, rows = _tokens(c, seed)
    if c["op"] == "write":
        out = {"k": [], "v": []}
        for b, (n, r) in enumerate(zip(lens, rows)):
            for name, t in (("k", k), ("v", v)):
                out[name].append(_exact_tokens(t[b], n + r, c["fmt"], c["closed"])[n // BLOCK * BLOCK:])
        return {name: torch.cat(parts) for name, parts in out.items()}
    starts, parts = _starts(rows), []
    for b, (n, r) in enumerate(zip(lens, rows)):
        tokens = n if c["closed"] else n + r
        raw = [t[b, :tokens].double().repeat_interleave(c["shared"], 1).transpose(0, 1) for t in (k, v)]
        held = [_exact_tokens(t[b], tokens, c["fmt"], c["closed"]).repeat_interleave(c["shared"], 1).transpose(0, 1) for t in (k, v)]
        if not c["closed"] and tokens % BLOCK:      # (the row behind the last token would read the last block as it is: so it stays)
            assert torch.equal(held[0][:, tokens // BLOCK * BLOCK:], raw[0][:, tokens // BLOCK * BLOCK:])
        qs = q[starts[b]:starts[b] + r].double().transpose(0, 1) / math.sqrt(c["width"])
        for lo in range(0, r, 64):
            t = torch.arange(n + lo, n + min(lo + 64, r), device="cuda")[:, None]
            key = torch.arange(tokens, device="cuda")[None, :]
            qq = qs[:, lo:lo + 64]
            x8 = qq @ held[0].transpose(1, 2)
            if c["closed"]:
                parts.append((torch.softmax(x8, -1) @ held[1]).transpose(0, 1))
                continue
            mine = key // BLOCK == t // BLOCK
            x = torch.where(mine, qq @ raw[0].transpose(1, 2), x8)
            w = torch.softmax(torch.where(key <= t, x, -math.inf), -1)
            parts.append((torch.where(mine, 0.0, w) @ held[1] + torch.where(mine, w, 0.0) @ raw[1]).transpose(0, 1))
    return torch.cat(parts)


def _exact_accept(c, seed):
    s = _scores(c, seed)
    at, draft = s["row_start"].tolist(), s["draft"].tolist()
    u, picks = s["accept_u"].tolist(), s["pick_u"].tolist()
    accepted, tokens = [], []
    for b in range(c["batch"]):
        got = []
        for r in range(at[b], at[b + 1]):
            log_p = torch.log_softmax(s["logits"][r].double() / float(s["temperature"][b]), 0)
            p, d = torch.exp(log_p), draft[r]
            drafted = torch.zeros_like(p)
            drafted[d] = 1.0
            if c["drafter"]:
                drafted = s["probs"][r].double()
            if u[r] * float(drafted[d]) < float(p[d]):
                got.append(d)
                continue
            left = torch.relu(p - drafted)
            sums = torch.cumsum(left, 0)
            got.append(int(torch.searchsorted(sums, picks[b] * sums[-1], right=True)) if float(sums[-1]) > 0 else d)
            break
        accepted.append(len(got))
        tokens += got + [-1] * (at[b + 1] - at[b] - len(got))
    return {"accepted": _i32(accepted), "tokens": _i32(tokens)}
