"""The library's operators that need no context, over torch tensors: key/value caches in 8 bits and the acceptance of sampled blocks.

Argument marshalling only, as in `binding`.  Work goes to torch's current stream of the tensors' device; row tables are int32 tensors
on that device, read when the kernels run, so the calls never wait and may be captured into graphs.  Workspaces come from torch's allocator
per call, which orders their reuse on the stream; two calls never share one.
"""
from __future__ import annotations

import ctypes as C
import math

from . import binding as B

_FORMATS = {"e4m3": B.AD_KV_E4M3, "i8": B.AD_KV_I8}


def _refuse(msg):
    raise B.AdError(B.AD_EINVAL, msg)


def _is(t, name, device, dtype, shape):
    import torch
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype != dtype or t.dim() != len(shape) or any(
            want is not None and got != want for got, want in zip(t.shape, shape)):
        _refuse(f"{name} must be a {dtype} tensor of shape {list(shape)} on {device}")
    return t


def _flat(t, name, device, dtype, shape):
    if not _is(t, name, device, dtype, shape).is_contiguous():
        _refuse(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(t, name, device, heads, width, rows=None):
    """Address and row stride of [rows, heads, width] bf16: rows may lie apart, a row's heads side by side."""
    import torch
    _is(t, name, device, torch.bfloat16, (rows, heads, width))
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != width):
        _refuse(f"{name}: the heads of a row must lie side by side")
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else heads * width)


class _On:
    """The device of a call: current for its length, its stream."""

    def __init__(self, device):
        import torch
        self.guard = None if torch.cuda.current_device() == device.index else torch.cuda.device(device)

    def __enter__(self):
        import torch
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream().cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)
        return False


class Kv8Cache:
    """Keys and values of `n_seq` sequences in 8 bits with a scale for each block of 32 tokens and head (include/ad.h, "key/value caches
    in 8 bits"), in device memory of its own.

    A growing cache is appended to and read as tokens come; a row reads its own block of 32 tokens in bf16 and every earlier one in
    8 bits, so results do not depend on how many tokens came in a call.  A closed one (an encoder's memory) is written once.

    `row_start` [n_seq + 1] and `length` [n_seq] are int32 tensors on the device: sequence b has the packed rows row_start[b] ..
    row_start[b + 1] - 1, at positions length[b] ..  Taking tokens back is passing a smaller length: any since the start of the last
    append, or a multiple of 32.  `max_rows` (the longest sequence's rows, default: all, at most k_max) and `max_keys` (default: the capacity)
    bound the launch; what the tables say beyond them is left out.
    """

    def __init__(self, n_seq, n_heads, head_width, capacity, k_max=1, format="e4m3", closed=False, device="cuda"):
        import torch
        if format not in _FORMATS:
            _refuse("format must be 'e4m3' or 'i8'")
        self.cfg = B.AdKv8Config(n_seq, n_heads, head_width, capacity, k_max, _FORMATS[format], int(bool(closed)))
        self._cfg = C.byref(self.cfg)
        self.L = B.lib()
        B._check(self.L.ad_kv8_check(self._cfg))
        self.most_rows = capacity if closed else k_max
        device = torch.device(device)
        self.device = torch.device("cuda", torch.cuda.current_device()) if device.index is None else device
        self.memory = torch.empty(self.L.ad_kv8_bytes(self._cfg), dtype=torch.uint8, device=self.device)

    def _tables(self, row_start, length, name="length"):
        import torch
        n = self.cfg.n_seq
        return (_flat(row_start, "row_start", self.device, torch.int32, (n + 1,)), _flat(length, name, self.device, torch.int32, (n,)))

    def append(self, k, v, row_start, length, max_rows=None):
        """Rows k, v [rows, n_heads, head_width] bf16 become the tokens from length[b] on."""
        c = self.cfg
        kp, ks = _rows(k, "k", self.device, c.n_heads, c.head_width)
        vp, vs = _rows(v, "v", self.device, c.n_heads, c.head_width, k.shape[0])
        start, at = self._tables(row_start, length)
        rows = k.shape[0]
        with _On(self.device) as stream:
            B._check(self.L.ad_kv8_append(self._cfg, self.memory.data_ptr(), kp, ks, vp, vs, start, at, rows,
                                          min(rows, self.most_rows) if max_rows is None else max_rows, stream))

    def read(self, row_start, begin, length, rows, max_rows=None, dtype=None):
        """The values the cache stands for, (k, v) [rows, n_heads, head_width]: tokens begin[b] .. of sequence b, as the row at position
        length[b] reads them, in packed rows row_start[b] ..; fp32 (exact) or bf16 (default)."""
        import torch
        dtype = torch.bfloat16 if dtype is None else dtype
        if dtype not in (torch.bfloat16, torch.float32):
            _refuse("dtype must be bfloat16 or float32")
        start, first = self._tables(row_start, begin, "begin")
        at = self._tables(row_start, length)[1]
        c = self.cfg
        with _On(self.device) as stream:
            k, v = (torch.empty((rows, c.n_heads, c.head_width), dtype=dtype, device=self.device) for _ in range(2))
            B._check(self.L.ad_kv8_read(self._cfg, self.memory.data_ptr(), start, first, at, rows, rows if max_rows is None else max_rows,
                                        B.AD_F32 if dtype == torch.float32 else B.AD_BF16, k.data_ptr(), v.data_ptr(), stream))
        return k, v

    def attend(self, q, row_start, length, max_rows=None, max_keys=None, scale=None, out=None):
        """softmax(scale q k^T) v of rows q [rows, q_heads, head_width] bf16 (appended before: at positions length[b] ..; closed: over length[b]
        tokens).  q_heads: a multiple of n_heads, neighbours share a head.  scale: 1 / sqrt(head_width) by default."""
        import torch
        c = self.cfg
        if not isinstance(q, torch.Tensor) or q.dim() != 3:
            _refuse("q must be a tensor [rows, q_heads, head_width]")
        rows, heads = q.shape[0], q.shape[1]
        qp, qs = _rows(q, "q", self.device, heads, c.head_width)
        start, at = self._tables(row_start, length)
        most = rows if c.closed else min(rows, c.k_max)
        keys = c.capacity if max_keys is None else max_keys
        with _On(self.device) as stream:
            if out is None:
                out = torch.empty((rows, heads, c.head_width), dtype=torch.bfloat16, device=self.device)
            op, os = _rows(out, "out", self.device, heads, c.head_width, rows)
            need = self.L.ad_kv8_attend_bytes(self._cfg, heads, rows, keys)
            ws = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
            B._check(self.L.ad_kv8_attend(self._cfg, self.memory.data_ptr(), qp, qs, heads, start, at, rows, most if max_rows is None else max_rows,
                                          keys, 1.0 / math.sqrt(c.head_width) if scale is None else scale, op, os,
                                          ws.data_ptr() if ws is not None else None, need, stream))
        return out


def accept_sampled(logits, draft, row_start, accept_u, pick_u, temperature=None, draft_probs=None, max_rows=None):
    """Verification of drafted tokens for sampled decoding (include/ad.h, "acceptance of sampled blocks"): (n_accept [n_seq], tokens [rows]).

    logits [rows, vocab] fp32 or bf16 (rows may lie apart), draft [rows] int32 (AD_NEVER: none), row_start [n_seq + 1] int32, accept_u [rows] and pick_u [n_seq]
    fp32 uniform in [0, 1), temperature [n_seq] fp32 or None (1), draft_probs [rows, vocab] fp32 or None (drafted tokens are certain)."""
    import torch
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or logits.dtype not in (torch.float32, torch.bfloat16) or logits.device.type != "cuda":
        _refuse("logits must be a float32 or bfloat16 tensor [rows, vocab] on a GPU")
    dev, (rows, vocab) = logits.device, logits.shape
    if vocab > 1 and logits.stride(1) != 1:
        _refuse("logits: a row's scores must lie side by side")
    f32, i32 = torch.float32, torch.int32
    if not isinstance(pick_u, torch.Tensor):
        _refuse("pick_u must be a tensor")
    n_seq = pick_u.shape[0] if pick_u.dim() == 1 else -1
    probs, probs_stride = None, 0
    if draft_probs is not None:
        _is(draft_probs, "draft_probs", dev, f32, (rows, vocab))
        if vocab > 1 and draft_probs.stride(1) != 1:
            _refuse("draft_probs: a row's probabilities must lie side by side")
        probs, probs_stride = draft_probs.data_ptr(), draft_probs.stride(0) if rows > 1 else vocab
    args = (_flat(accept_u, "accept_u", dev, f32, (rows,)), _flat(pick_u, "pick_u", dev, f32, (n_seq,)),
            _flat(row_start, "row_start", dev, i32, (n_seq + 1,)))
    drafted = _flat(draft, "draft", dev, i32, (rows,))
    temp = None if temperature is None else _flat(temperature, "temperature", dev, f32, (n_seq,))
    L = B.lib()
    with _On(dev) as stream:
        n_accept = torch.empty(n_seq, dtype=i32, device=dev)
        tokens = torch.empty(rows, dtype=i32, device=dev)
        need = L.ad_accept_sampled_bytes(n_seq, rows, vocab)
        ws = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)
        B._check(L.ad_accept_sampled(logits.data_ptr(), B.AD_F32 if logits.dtype == f32 else B.AD_BF16, logits.stride(0) if rows > 1 else vocab, vocab,
                                     drafted, probs, probs_stride, temp, *args, n_seq, rows, rows if max_rows is None else max_rows,
                                     n_accept.data_ptr(), tokens.data_ptr(), ws.data_ptr(), need, stream))
    return n_accept, tokens
