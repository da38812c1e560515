"""KVBatch: serving steps on a pool's resident KV (include/lv.h, "a serving step on resident KV").

A step takes new tokens of several sessions -- single tokens of a reply, chunks of user input, or
both -- whose room in the context a turn or ``KVPool.append`` has made:

    batch = KVBatch(pool, q_heads=32, max_requests=64, max_tokens=4096)
    batch.plan(sids, lens)                       # once a step: tables, positions, slot map
    for layer in range(pool.L):                  # q, k, v: [rows, heads, head_dim]
        batch.write(layer, k, v)
        out = batch.attention(layer, q)

``row_starts``, ``kv_lens``, ``tables``, ``positions`` and ``slots`` are device tensors that
``plan`` fills.  A captured ``write`` or ``attention`` works on the step planned last when it is replayed;
it keeps the rows and the attention's kernel (chosen from the rows a request) of the plan before its
capture, and does nothing but report LV_ERR_STATE where a later plan has more rows or the other kernel:
plan with the same ``num_tokens`` and ``max_len`` each time.  PyTorch holds the memory; every operation is a liblv call on the given stream (None:
the pool's, or the current one).
"""
from __future__ import annotations

import math

import numpy as np
import torch

from . import lv
from .pool import KVPool

_PLAN_ONE_LAUNCH = 256         # requests up to which a plan is one kernel
_KINDS = {torch.bfloat16: lv.LV_BF16, torch.float16: lv.LV_F16, torch.float32: lv.LV_F32}


class KVBatch:
    """One kind of attention layer over ``pool``: ``q_heads`` query heads, and with ``window`` > 0 a
    sliding window of that many keys beside which the first ``sinks`` keys stay visible.

    It holds device memory until ``close`` or the pool's: the library's workspace and work lists, and
    the five arrays, of which ``tables`` has max_requests * max_blocks entries."""

    def __init__(self, pool: KVPool, *, q_heads: int, max_requests: int, max_tokens: int,
                 dtype=torch.bfloat16, window: int = 0, sinks: int = 0):
        if dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("dtype must be torch.bfloat16 or torch.float16")
        self.pool, self.q_heads, self.dtype = pool, q_heads, dtype
        self.max_requests, self.max_tokens = max_requests, max_tokens
        self.num_tokens = 0
        self.handle = None
        i32 = dict(dtype=torch.int32, device=pool.device)
        rows, requests = max(max_tokens, 0), max(max_requests, 0)
        with torch.cuda.device(pool.device):
            self.row_starts = torch.zeros(requests + 1, **i32)
            self.kv_lens = torch.zeros(max(requests, 1), **i32)
            self.tables = torch.full((max(requests, 1), pool.max_blocks), -1, **i32)
            self.positions = torch.full((max(rows, 1),), -1, **i32)
            self.slots = torch.full((max(rows, 1),), -1, dtype=torch.int64, device=pool.device)
            # the library may write them on any stream next
            torch.cuda.current_stream().synchronize()
        self._device = self.row_starts.get_device()
        self._used_on = {lv.stream_handle(None, self._device)}      # streams that keep the arrays above in use
        self._scale = 1.0 / math.sqrt(pool.head_dim)
        self._a, self._b = lv.lv_heads(), lv.lv_heads()      # a call's two tensor arguments
        # an output that attention() makes itself
        self._own = lv.lv_heads(row_stride=q_heads * pool.head_dim, head_stride=pool.head_dim,
                                dtype=_KINDS[dtype])
        d = lv.lv_batch_desc(num_q_heads=q_heads, max_requests=max_requests, max_tokens=max_tokens,
                             dtype=_KINDS[dtype], window=window, sinks=sinks,
                             row_starts=self.row_starts.data_ptr(), kv_lens=self.kv_lens.data_ptr(),
                             tables=self.tables.data_ptr(), positions=self.positions.data_ptr(),
                             slots=self.slots.data_ptr())
        self.handle = lv.lv_batch_create(pool.handle, d)
        pool.attach(self)          # destroyed before the pool

    def close(self):
        """Waits for the pool's stream (or the current one) and frees the batch's memory; what is
        captured over it cannot be replayed any more."""
        if getattr(self, "handle", None):
            lv.lv_batch_destroy(self.handle, self.pool.stream)
            self.handle = None
            self.row_starts = self.kv_lens = self.tables = self.positions = self.slots = None
            self.pool.detach(self)

    def _ints(self, x, n=None):
        """An int32 array the library can read: a tensor as it is, else a numpy array."""
        if isinstance(x, torch.Tensor):
            if x.dtype is not torch.int32 or not x.is_contiguous():
                raise ValueError("expected a contiguous int32 tensor")
            if x.is_cuda and x.get_device() != self._device:
                raise ValueError("expected a tensor on the pool's device")
        else:
            x = np.ascontiguousarray(x, dtype=np.int32)
        if n is not None and len(x) != n:
            raise ValueError(f"expected {n} entries, got {len(x)}")
        return x

    def plan(self, sids, lens, firsts=None, *, num_tokens=None, max_len=None, stream=None):
        """Plans a step: request i is session sids[i] with lens[i] new tokens from position firsts[i]
        on (None: the last ones of its context).  With lengths on the device, ``num_tokens`` (rows of
        the step's tensors) has to be given, and ``max_len`` (a bound of the lengths) should be."""
        sids = self._ints(sids)
        n = len(sids)
        lens = self._ints(lens, n)
        if firsts is not None:
            firsts = self._ints(firsts, n)
        if isinstance(lens, torch.Tensor) and lens.is_cuda:
            if num_tokens is None:
                raise ValueError("num_tokens is needed with lengths on the device")
        elif num_tokens is None or max_len is None:
            have = np.asarray(lens)
            num_tokens = int(have.sum()) if num_tokens is None else num_tokens
            max_len = int(have.max(initial=0)) if max_len is None else max_len
        s, away = self._stream(stream)
        if away or s not in self._used_on:
            self._use(s, sids, lens, firsts)
        lv.lv_batch_plan(self.handle, sids, firsts, lens, n, num_tokens,
                         num_tokens if max_len is None else max_len, s)
        self.num_tokens = num_tokens
        self.pool.launches += 1 + (n > _PLAN_ONE_LAUNCH)

    def _stream(self, stream):
        """The handle of a call's stream, and whether it is another than the current one."""
        if stream is None:
            stream = self.pool.stream
        s = lv.stream_handle(stream, self._device)
        return s, stream is not None and s != lv.stream_handle(None, self._device)

    def _torch_stream(self, s):
        return torch.cuda.ExternalStream(s, device=self.pool.device) if s else \
            torch.cuda.default_stream(self.pool.device)

    def _use(self, s, *tensors):
        """Before a launch on the stream of handle s: PyTorch gives no memory that the launch uses to
        others before it has run.  (On the current stream that holds for a call's own tensors already.)"""
        t = self._torch_stream(s)
        if s not in self._used_on:
            self._used_on.add(s)
            tensors += (self.row_starts, self.kv_lens, self.tables, self.positions, self.slots)
        for x in tensors:
            if isinstance(x, torch.Tensor) and x.is_cuda:
                x.record_stream(t)

    def _put(self, h, x, heads, name):
        """h describes tensor x, [rows, heads, head_dim] with head_dim contiguous."""
        shape, (row, head, last) = x.shape, x.stride() if x.dim() == 3 else (0, 0, 0)
        if len(shape) != 3 or shape[0] < self.num_tokens or shape[1] != heads or \
                shape[2] != self.pool.head_dim or last != 1 or x.dtype not in _KINDS or \
                x.get_device() != self._device:
            raise ValueError(f"{name}: expected a bf16, f16 or f32 tensor [{self.num_tokens}, {heads}, "
                             f"{self.pool.head_dim}] on {self.pool.device} with contiguous head_dim, got "
                             f"{tuple(shape)} of {x.dtype} on {x.device}")
        h.data, h.row_stride, h.head_stride, h.dtype = x.data_ptr(), row, head, _KINDS[x.dtype]
        return h

    def write(self, layer: int, k, v, *, stream=None):
        """The step's new K and V rows ([rows, kv_heads, head_dim], any strides, bf16, f16 or f32)
        into their pages."""
        H = self.pool.kv_heads
        s, away = self._stream(stream)
        k_arg, v_arg = self._put(self._a, k, H, "k"), self._put(self._b, v, H, "v")
        if away or s not in self._used_on:
            self._use(s, k, v)
        lv.lv_kv_write(self.handle, layer, k_arg, v_arg, s)
        self.pool.launches += 1

    def attention(self, layer: int, q, *, out=None, scale=None, return_lse=False, stream=None):
        """Attention of the step's rows over their paged contexts: [rows, q_heads, head_dim], and with
        ``return_lse`` the logarithms of the sums of exponentials [rows, q_heads] (f32).  Rows of
        no request give zeros (and -inf).  scale: 1 / sqrt(head_dim) unless given.  With a stream
        other than the current one, the caller orders the two: the stream after what made q, and what
        reads the results after the stream."""
        s, away = self._stream(stream)
        if away or s not in self._used_on:
            self._use(s, q, out)
        if away:
            # results from the launch's own stream: the current one's memory may be in use there
            with torch.cuda.stream(self._torch_stream(s)):
                made = self.attention(layer, q, out=out, scale=scale, return_lse=return_lse, stream=s)
            for x in made if return_lse else (made,):
                x.record_stream(torch.cuda.current_stream(self.pool.device))
            return made
        q_arg = self._put(self._a, q, self.q_heads, "q")
        lse = None
        if out is None:
            out = torch.empty_like(q) if q.is_contiguous() and q.dtype is self.dtype else \
                torch.empty(q.shape, dtype=self.dtype, device=q.device)
            out_arg = self._own
            out_arg.data = out.data_ptr()
            if len(out) > self.num_tokens:       # rows that the step does not have
                out[self.num_tokens:].zero_()
        else:
            out_arg = self._put(self._b, out, self.q_heads, "out")
        if return_lse:
            lse = torch.empty((len(q), self.q_heads), dtype=torch.float32, device=q.device)
            if len(q) > self.num_tokens:
                lse[self.num_tokens:].fill_(-math.inf)
        lv.lv_attention(self.handle, layer, q_arg, out_arg, lse, self._scale if scale is None else scale, s)
        self.pool.launches += 1
        return (out, lse) if return_lse else out
