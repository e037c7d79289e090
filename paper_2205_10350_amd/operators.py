"""The library's operators that need no context, over torch tensors: key/value caches in 8 bits, the acceptance of sampled blocks, and distributions cut by
top-k, top-p and min-p.

Argument marshalling only, as in `binding`.  Work goes to torch's current stream of the tensors' device; row tables are int32 tensors
on that device, read when the kernels run, so the calls never wait and may be captured into graphs.  Workspaces come from torch's allocator
per call, which orders their reuse on the stream; two calls never share one.
"""
from __future__ import annotations

import ctypes as C
import functools
import math

from . import binding as B

_FORMATS = {"e4m3": B.AD_KV_E4M3, "i8": B.AD_KV_I8}


def _refuse(msg):
    raise B.AdError(B.AD_EINVAL, msg)


# The checks of a call are most of what the smallest calls cost: plain comparisons, one pass, words only where one fails.
def _flat(t, name, index, dtype, shape):
    """Address of a contiguous tensor of that type and shape on GPU `index`."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _refuse(f"{name} must be a contiguous {dtype} tensor of shape {list(shape)} on cuda:{index}")


def _rows(t, name, index, dtype, heads, width):
    """Address, row stride and rows of [rows, heads, width]: rows may lie apart, a row's heads side by side."""
    try:
        rows, h, w = t.shape
        if t.dtype is dtype and h == heads and w == width and t.get_device() == index:
            apart, side, one = t.stride()
            if one == 1 and (side == width or h == 1):
                return t.data_ptr(), (apart if rows > 1 else h * w), rows
    except (AttributeError, ValueError):
        pass
    _refuse(f"{name} must be a {dtype} tensor [rows, {heads}, {width}] on cuda:{index}, the heads of a row side by side")


def _count(name, n):
    if not -2**31 <= n < 2**31:
        _refuse(f"{name}: {n} is no 32-bit number")
    return n


def _bound(max_rows, rows):
    """max_rows as the call takes it: no sequence has more than all rows."""
    return min(_count("max_rows", max_rows), rows)


def _on(index, call):
    """call(stream) with GPU `index` current and its current stream."""
    import torch
    if torch._C._cuda_getDevice() == index:
        return call(torch._C._cuda_getCurrentRawStream(index))
    with torch.cuda.device(index):
        return call(torch._C._cuda_getCurrentRawStream(index))


class Kv8Cache:
    """Keys and values of `n_seq` sequences in 8 bits with a scale for each block of 32 tokens and head (include/ad.h, "key/value caches
    in 8 bits"), in device memory of its own.

    A growing cache is appended to and read as tokens come; a row reads its own block of 32 tokens in bf16 and every earlier one in
    8 bits, so results do not depend on how many tokens came in a call.  A closed one (an encoder's memory) is written once.

    `row_start` [n_seq + 1] and `length` [n_seq] are int32 tensors on the device: sequence b has the packed rows row_start[b] ..
    row_start[b + 1] - 1, at positions length[b] ..  Taking tokens back is passing a smaller length: any since the start of the last
    append, or a multiple of 32.  `max_rows` (at least the longest sequence's rows) and `max_keys` (default: the capacity) bound the launch; what the tables say
    beyond them is left out.  Without `max_rows` a sequence may have k_max rows in a call (closed: the capacity): the tables are read on the device, so it is the caller's to
    see that none has more, whose rows would be left out.  More packed rows than all sequences together may have are refused: some would be
    left out, or lie behind the last sequence, and then `max_rows` says that this is meant.
    """

    def __init__(self, n_seq, n_heads, head_width, capacity, k_max=1, format="e4m3", closed=False, device="cuda"):
        import torch
        if format not in _FORMATS:
            _refuse("format must be 'e4m3' or 'i8'")
        for n in (n_seq, n_heads, head_width, capacity, k_max):
            _count("the cache's sizes", n)
        self.cfg = B.AdKv8Config(n_seq, n_heads, head_width, capacity, k_max, _FORMATS[format], int(bool(closed)))
        self._cfg = C.byref(self.cfg)
        self.L = B.lib()
        B._check(self.L.ad_kv8_check(self._cfg))
        self.most_rows = capacity if closed else k_max
        device = torch.device(device)
        if device.type != "cuda":
            _refuse("the cache must be on a GPU")
        self.index = torch.cuda.current_device() if device.index is None else device.index
        self.device = torch.device("cuda", self.index)
        self.memory = torch.empty(self.L.ad_kv8_bytes(self._cfg), dtype=torch.uint8, device=self.device)
        self._streams = {torch.cuda.current_stream(self.device).cuda_stream}
        self._at = self.memory.data_ptr()
        self._start, self._len = (n_seq + 1,), (n_seq,)
        self._i32, self._bf16 = torch.int32, torch.bfloat16
        self._scale = 1.0 / math.sqrt(head_width)
        self._need = {}

    def _used_on(self, stream):
        if stream not in self._streams:   # (the allocator is to wait for that stream, too, before it gives the memory to others)
            import torch
            self.memory.record_stream(torch.cuda.current_stream(self.device))
            self._streams.add(stream)

    def _call(self, call, other=None):
        def on(stream):
            self._used_on(stream)
            if other is not None:
                other._used_on(stream)
            return call(stream)
        rc = _on(self.index, on)
        if rc:
            B._check(rc)

    def _most(self, rows):
        if rows > self.cfg.n_seq * self.most_rows:
            _refuse(f"{rows} rows, where {self.cfg.n_seq} sequence(s) may have {self.most_rows} each in a call: pass max_rows if rows lie behind the last sequence")
        return min(rows, self.most_rows)

    def append(self, k, v, row_start, length, max_rows=None):
        """Rows k, v [rows, n_heads, head_width] bf16 become the tokens from length[b] on."""
        c, i = self.cfg, self.index
        kp, ks, rows = _rows(k, "k", i, self._bf16, c.n_heads, c.head_width)
        vp, vs, vrows = _rows(v, "v", i, self._bf16, c.n_heads, c.head_width)
        if vrows != rows:
            _refuse("k and v must have as many rows")
        start, at = _flat(row_start, "row_start", i, self._i32, self._start), _flat(length, "length", i, self._i32, self._len)
        most = self._most(rows) if max_rows is None else _bound(max_rows, rows)
        self._call(lambda stream: self.L.ad_kv8_append(self._cfg, self._at, kp, ks, vp, vs, start, at, rows, most, stream))

    def read(self, row_start, begin, length, rows, max_rows=None, dtype=None):
        """The values the cache stands for, (k, v) [rows, n_heads, head_width]: tokens begin[b] .. of sequence b, as the row at position
        length[b] reads them, in packed rows row_start[b] ..; fp32 (exact) or bf16 (default)."""
        import torch
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in (torch.bfloat16, torch.float32):
            _refuse("dtype must be bfloat16 or float32")
        c, i = self.cfg, self.index
        _count("rows", rows)
        start, first = _flat(row_start, "row_start", i, self._i32, self._start), _flat(begin, "begin", i, self._i32, self._len)
        at = _flat(length, "length", i, self._i32, self._len)
        k = torch.empty((rows, c.n_heads, c.head_width), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        kp, vp = k.data_ptr(), v.data_ptr()
        most = rows if max_rows is None else _bound(max_rows, rows)
        kind = B.AD_F32 if dtype is torch.float32 else B.AD_BF16
        self._call(lambda stream: self.L.ad_kv8_read(self._cfg, self._at, start, first, at, rows, most, kind, kp, vp, stream))
        return k, v

    def attend(self, q, row_start, length, max_rows=None, max_keys=None, scale=None, out=None):
        """softmax(scale q k^T) v of rows q [rows, q_heads, head_width] bf16 (appended before: at positions length[b] ..; closed: over length[b]
        tokens).  q_heads: a multiple of n_heads, neighbours share a head.  scale: 1 / sqrt(head_width) by default."""
        import torch
        c, i = self.cfg, self.index
        heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
        qp, qs, rows = _rows(q, "q", i, self._bf16, heads, c.head_width)
        start, at = _flat(row_start, "row_start", i, self._i32, self._start), _flat(length, "length", i, self._i32, self._len)
        most = (rows if c.closed else self._most(rows)) if max_rows is None else _bound(max_rows, rows)
        keys = c.capacity if max_keys is None else min(max_keys, c.capacity)
        scale = self._scale if scale is None else scale

        def call(stream):
            nonlocal out
            if out is None and qs == heads * c.head_width:
                out = torch.empty_like(q)
                op, os = out.data_ptr(), qs
            else:
                if out is None:
                    out = torch.empty((rows, heads, c.head_width), dtype=self._bf16, device=self.device)
                op, os, orows = _rows(out, "out", i, self._bf16, heads, c.head_width)
                if orows != rows:
                    _refuse("out must have as many rows as q")
            need = self._need.get((heads, rows, keys))
            if need is None:
                if len(self._need) >= 4096:
                    self._need.clear()
                need = self._need[heads, rows, keys] = self.L.ad_kv8_attend_bytes(self._cfg, heads, rows, keys)
            # (held until the kernels are enqueued; whatever gets it from the allocator afterwards comes behind them on this stream)
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            return self.L.ad_kv8_attend(self._cfg, self._at, qp, qs, heads, start, at, rows, most, keys, scale, op, os,
                                        None if ws is None else ws.data_ptr(), need, stream)
        self._call(call)
        return out

    def attend_shared(self, q, row_start, length, shared, seq_start, shared_length, max_rows=None, max_keys=None, max_shared_rows=None,
                      max_shared_keys=None, scale=None, out=None):
        """`attend` of rows whose sequences share texts: softmax over the text's tokens and the sequence's own up to the row, what texts hold being read once for all of
        their sequences.  `shared`: a cache of the same heads and format (this one, too) with a text a sequence, the first shared_length[g] tokens of sequence g
        (int32 [shared.n_seq]; of a growing cache whole blocks of 32, all in 8 bits).  Text g belongs to this cache's sequences seq_start[g] .. seq_start[g + 1] - 1 (int32 [shared.n_seq + 1],
        ascending), which lie next to each other; sequences of no text see their own tokens alone.  Positions and `length` count a sequence's own tokens.  max_shared_rows:
        at least the most rows of a text's sequences together (default: all); max_shared_keys: at least the longest text (default: the capacity)."""
        import torch
        c, i = self.cfg, self.index
        if not isinstance(shared, Kv8Cache) or shared.index != i:
            _refuse(f"shared must be a Kv8Cache on cuda:{i}")
        heads = q.shape[1] if isinstance(q, torch.Tensor) and q.dim() == 3 else 0
        qp, qs, rows = _rows(q, "q", i, self._bf16, heads, c.head_width)
        start, at = _flat(row_start, "row_start", i, self._i32, self._start), _flat(length, "length", i, self._i32, self._len)
        first, texts = _flat(seq_start, "seq_start", i, self._i32, shared._start), _flat(shared_length, "shared_length", i, self._i32, shared._len)
        most = self._most(rows) if max_rows is None else _bound(max_rows, rows)
        together = rows if max_shared_rows is None else min(_count("max_shared_rows", max_shared_rows), rows)
        keys = c.capacity if max_keys is None else min(_count("max_keys", max_keys), c.capacity)
        text_keys = shared.cfg.capacity if max_shared_keys is None else min(_count("max_shared_keys", max_shared_keys), shared.cfg.capacity)
        scale = self._scale if scale is None else scale

        def call(stream):
            nonlocal out
            if out is None and qs == heads * c.head_width:
                out = torch.empty_like(q)
                op, os = out.data_ptr(), qs
            else:
                if out is None:
                    out = torch.empty((rows, heads, c.head_width), dtype=self._bf16, device=self.device)
                op, os, orows = _rows(out, "out", i, self._bf16, heads, c.head_width)
                if orows != rows:
                    _refuse("out must have as many rows as q")
            sizes = heads, rows, keys, text_keys, shared.cfg.n_seq, shared.cfg.capacity
            need = self._need.get(sizes)
            if need is None:
                if len(self._need) >= 4096:
                    self._need.clear()
                need = self._need[sizes] = self.L.ad_kv8_attend_shared_bytes(self._cfg, shared._cfg, heads, rows, keys, text_keys)
            # (held until the kernels are enqueued; whatever gets it from the allocator afterwards comes behind them on this stream)
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            return self.L.ad_kv8_attend_shared(self._cfg, self._at, shared._cfg, shared._at, qp, qs, heads, start, at, first, texts, rows, most, keys, together, text_keys,
                                               scale, op, os, None if ws is None else ws.data_ptr(), need, stream)
        self._call(call, shared)
        return out

    def copy(self, source, place, end, begin=None, origin=None, max_tokens=None):
        """Sequences forked, moved together or taken over from another cache: the first end[i] tokens of sequence source[i] of `origin` (a cache of the same heads and format;
        default: this one) become those of this cache's sequence place[i], as if all were read before any is written.  source, place, end: int32 [n] on the device.  `begin`
        (int32 [n], multiples of 32, from another cache only): tokens begin[i] .. end[i] - 1 become the first ones.  end[i] is any length that the source may be taken back to.  Of
        entries with one place the first counts (also if it has no tokens); what lies outside the caches is left out.  `max_tokens`: at least the most tokens of an entry (default: the capacity).  A growing cache's
        copy that this or the capacity cuts short inside one of the source's complete blocks ends with the block before."""
        i = self.index
        if origin is not None and (not isinstance(origin, Kv8Cache) or origin.index != i):
            _refuse(f"origin must be a Kv8Cache on cuda:{i}")
        n = (source.shape[0],) if hasattr(source, "shape") and len(source.shape) == 1 else (-1,)
        sp, pp, ep = (_flat(t, name, i, self._i32, n) for t, name in ((source, "source"), (place, "place"), (end, "end")))
        bp = None if begin is None else _flat(begin, "begin", i, self._i32, n)
        o = self if origin is None else origin
        most = self.cfg.capacity if max_tokens is None else min(_count("max_tokens", max_tokens), self.cfg.capacity)
        self._call(lambda stream: self.L.ad_kv8_copy(o._cfg, o._at, self._cfg, self._at, sp, pp, bp, ep, n[0], most, stream), origin)


def accept_sampled(logits, draft, row_start, accept_u, pick_u, temperature=None, draft_probs=None, max_rows=None):
    """Verification of drafted tokens for sampled decoding (include/ad.h, "acceptance of sampled blocks"): (n_accept [n_seq], tokens [rows]).

    logits [rows, vocab] fp32 or bf16 (rows may lie apart), draft [rows] int32 (AD_NEVER: none), row_start [n_seq + 1] int32, accept_u [rows] and pick_u [n_seq]
    fp32 uniform in [0, 1), temperature [n_seq] fp32 or None (1), draft_probs [rows, vocab] fp32 or None (drafted tokens are certain),
    max_rows: at least the longest sequence's rows (default: all)."""
    import torch
    f32, i32 = torch.float32, torch.int32
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in (f32, torch.bfloat16) or not logits.is_cuda:
        _refuse("logits must be a float32 or bfloat16 tensor [rows, vocab] on a GPU")
    i, (rows, vocab), (stride, one) = logits.get_device(), logits.shape, logits.stride()
    if vocab > 1 and one != 1:
        _refuse("logits: a row's scores must lie side by side")
    n_seq = pick_u.shape[0] if isinstance(pick_u, torch.Tensor) and pick_u.dim() == 1 else -1
    probs, probs_stride = None, 0
    if draft_probs is not None:
        if not isinstance(draft_probs, torch.Tensor) or draft_probs.dtype is not f32 or draft_probs.shape != logits.shape or draft_probs.get_device() != i:
            _refuse(f"draft_probs must be a float32 tensor {[rows, vocab]} on cuda:{i}")
        probs, (probs_stride, one) = draft_probs.data_ptr(), draft_probs.stride()
        if vocab > 1 and one != 1:
            _refuse("draft_probs: a row's probabilities must lie side by side")
    drafted = _flat(draft, "draft", i, i32, (rows,))
    u, v = _flat(accept_u, "accept_u", i, f32, (rows,)), _flat(pick_u, "pick_u", i, f32, (n_seq,))
    start = _flat(row_start, "row_start", i, i32, (n_seq + 1,))
    temp = None if temperature is None else _flat(temperature, "temperature", i, f32, (n_seq,))
    n_accept, tokens = torch.empty_like(pick_u, dtype=i32), torch.empty_like(draft)
    need = _accept_bytes(n_seq, rows, vocab)

    def call(stream):
        # (held until the kernels are enqueued; whatever gets it from the allocator afterwards comes behind them on this stream)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=logits.device)
        return B.lib().ad_accept_sampled(logits.data_ptr(), B.AD_F32 if logits.dtype is f32 else B.AD_BF16, stride if rows > 1 else vocab, vocab,
                                         drafted, probs, probs_stride if rows > 1 else vocab, temp, u, v, start, n_seq, rows,
                                         rows if max_rows is None else _bound(max_rows, rows), n_accept.data_ptr(), tokens.data_ptr(), ws.data_ptr(), need, stream)
    rc = _on(i, call)
    if rc:
        B._check(rc)
    return n_accept, tokens


@functools.lru_cache(maxsize=4096)
def _accept_bytes(n_seq, rows, vocab):
    return B.lib().ad_accept_sampled_bytes(n_seq, rows, vocab)


def _cut(logits, temperature, top_k, top_p, min_p, row_start):
    """What sample_tokens and truncate_scores have in common: the call's arguments up to the number of sequences, the GPU and the rows."""
    import torch
    f32, i32 = torch.float32, torch.int32
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in (f32, torch.bfloat16) or not logits.is_cuda:
        _refuse("logits must be a float32 or bfloat16 tensor [rows, vocab] on a GPU")
    i, (rows, vocab), (stride, one) = logits.get_device(), logits.shape, logits.stride()
    if vocab > 1 and one != 1:
        _refuse("logits: a row's scores must lie side by side")
    n_seq, start = rows, None
    if row_start is not None:
        n_seq = row_start.shape[0] - 1 if isinstance(row_start, torch.Tensor) and row_start.dim() == 1 else -1
        start = _flat(row_start, "row_start", i, i32, (n_seq + 1,))
    cut = [None if t is None else _flat(t, name, i, dtype, (n_seq,))
           for t, name, dtype in ((temperature, "temperature", f32), (top_k, "top_k", i32), (top_p, "top_p", f32), (min_p, "min_p", f32))]
    return (logits.data_ptr(), B.AD_F32 if logits.dtype is f32 else B.AD_BF16, stride if rows > 1 else vocab, vocab, *cut, start, n_seq), i, rows


def sample_tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, row_start=None, log_probs=False):
    """Tokens drawn from truncated distributions by given random numbers (include/ad.h, "truncated distributions"): tokens [rows] int32, with log_probs=True also the
    logarithms of their probabilities [rows] fp32.

    logits [rows, vocab] fp32 or bf16 (rows may lie apart; a vocabulary of up to 2^20), u [rows] fp32 uniform in [0, 1).  temperature fp32, top_k int32, top_p fp32, min_p fp32: None or a tensor on the
    device with a setting for each row, or with row_start [n_seq + 1] int32 for each sequence, whose rows are row_start[b] .. row_start[b + 1] - 1."""
    import torch
    args, i, rows = _cut(logits, temperature, top_k, top_p, min_p, row_start)
    up = _flat(u, "u", i, torch.float32, (rows,))
    tokens = torch.empty_like(u, dtype=torch.int32)
    probs = torch.empty_like(u) if log_probs else None
    rc = _on(i, lambda stream: B.lib().ad_sample_tokens(*args, up, rows, tokens.data_ptr(), None if probs is None else probs.data_ptr(), stream))
    if rc:
        B._check(rc)
    return (tokens, probs) if log_probs else tokens


def truncate_scores(logits, temperature=None, top_k=None, top_p=None, min_p=None, row_start=None, out=None):
    """Scores without what top-k, top-p and min-p cut off: [rows, vocab] like logits, -inf in its place (include/ad.h, "truncated distributions").  With them as its logits, and the same
    temperature, `accept_sampled` verifies drafts against the truncated distributions.  Arguments as sample_tokens'; `out`: a tensor like logits that does not overlap it, or logits itself."""
    import torch
    args, i, rows = _cut(logits, temperature, top_k, top_p, min_p, row_start)
    vocab = logits.shape[1]
    if out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    elif not isinstance(out, torch.Tensor) or out.dtype is not logits.dtype or out.shape != logits.shape or out.get_device() != i or (vocab > 1 and out.stride(1) != 1):
        _refuse(f"out must be a {logits.dtype} tensor {[rows, vocab]} on cuda:{i}, a row's scores side by side")
    stride = out.stride(0) if rows > 1 else vocab
    rc = _on(i, lambda stream: B.lib().ad_truncate_scores(*args, rows, out.data_ptr(), stride, stream))
    if rc:
        B._check(rc)
    return out
