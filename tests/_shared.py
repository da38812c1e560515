"""A step whose requests continue prefixes that other sessions hold, and its attention in 64 bits."""
import numpy as np
import torch

from tests._attention import Step


class SharedStep(Step):
    """Request i continues the first ``plens[of[i]]`` (all, where plens is None) of prefix of[i]'s ``prefix``
    tokens, or none (-1).  The prefixes are further sessions of the step's pool."""

    def __init__(self, cached, new, of, prefix, plens=None, **kw):
        self.requests, self.of, self.prefix = len(new), list(of), list(prefix)
        self.plens = list(prefix if plens is None else plens)
        super().__init__(list(cached) + self.prefix, list(new) + [0] * len(prefix), **kw)
        from paper_2606_22983_gb300.batch import KVBatch
        self.batch.close()
        self.batch = KVBatch(self.pool, q_heads=self.heads * self.group, max_requests=max(self.requests, 1),
                             max_tokens=max(self.rows, 1), dtype=self.dtype, prefix_rows=max(self.rows, 1))
        self.given = plens is not None

    def psid(self, i):
        return int(self.sids[self.requests + self.of[i]]) if self.of[i] >= 0 else -1

    def plan(self, conv=lambda x: x, **kw):
        n = self.requests
        ints = lambda x: conv(np.asarray(x, np.int32))
        lens = [self.plens[p] if p >= 0 else 7 for p in self.of]        # (one that nobody has is not looked at)
        kw.setdefault("max_len", max(self.new, default=0))
        self.batch.plan(ints(self.sids[:n]), ints(self.new[:n]), prefixes=ints([self.psid(i) for i in range(n)]),
                        prefix_lens=ints(lens) if self.given else None, num_tokens=self.rows, **kw)

    def before(self, i):
        return self.plens[self.of[i]] if i < self.requests and self.of[i] >= 0 else 0

    def rows_of(self, i, kv, layer):
        x = super().rows_of(i, kv, layer)
        if self.before(i):
            x = torch.cat([super().rows_of(self.requests + self.of[i], kv, layer)[:self.before(i)], x])
        return x

    def seen(self, i):
        s = super().seen(i)
        return torch.cat([torch.ones((len(s), self.before(i)), dtype=torch.bool, device=s.device), s], 1)
