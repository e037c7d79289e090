"""The library's operators that need no context, over torch tensors: key/value caches in 8 bits and the acceptance of sampled blocks.

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

    def _call(self, call):
        def on(stream):
            if stream not in self._streams:   # (the allocator is to wait for that stream, too, before it gives the memory to others)
                import torch
                self.memory.record_stream(torch.cuda.current_stream(self.device))
                self._streams.add(stream)
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
