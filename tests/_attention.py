"""A pool with a serving step in it, and the step's operators in 64 bits on the host's arrays."""
import numpy as np
import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # unit roundoff


class Step:
    """Sessions of ``cached`` + ``new`` tokens over scattered pages.  Whatever no request's context
    holds is NaN: pages that nobody owns, and the rows of a last page past the context's end."""

    def __init__(self, cached, new, *, heads=2, group=4, dim=64, page=16, layers=2, dtype=torch.bfloat16,
                 window=0, sinks=0, pad=0, seed=0, spare=3, sharp=1.0, absent=(), host_pages=0, tiers=0,
                 max_requests=None, max_tokens=None):
        from paper_2606_22983_gb300.batch import KVBatch
        from paper_2606_22983_gb300.pool import KVPool
        rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.n = n = len(new)
        self.cached, self.new = list(cached), list(new)
        self.total = [a + b for a, b in zip(cached, new)]
        self.heads, self.group, self.dim, self.page, self.dtype = heads, group, dim, page, dtype
        self.window, self.sinks = window, sinks
        self.rows = sum(new) + pad
        sessions = 2 * n + 1
        self.sids = rng.permutation(sessions)[:n].astype(np.int32)
        blocks = [-(-t // page) for t in self.total]
        width = max(max(blocks, default=1), 1) + 1
        pages = sum(blocks) + spare
        kv = torch.full((2 * layers, pages, page, heads, dim), float("nan"), dtype=dtype, device="cuda")
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((sessions, width), -1, np.int32)
        ctx = np.zeros(sessions, np.int32)
        at = slot = 0
        for i, (sid, b, t) in enumerate(zip(self.sids, blocks, self.total)):
            self.table[sid, :b] = order[at:at + b]
            ctx[sid] = t
            for blk in range(b):
                p, rows = int(order[at + blk]), min(page, t - blk * page)
                kv[:, p, :rows] = torch.randn((2 * layers, rows, heads, dim), generator=self.gen, device="cuda",
                                              dtype=torch.float32).to(dtype)
                if (i, blk) in absent:                # in the host tier: its HBM page is nobody's
                    kv[:, p] = float("nan")
                    self.table[sid, blk] = -2 - slot
                    slot += 1
            at += b
        self.kv = kv
        self.pool = KVPool(layers=layers, kv_heads=heads, head_dim=dim, page_tokens=page, max_sessions=sessions,
                           max_blocks=width, hbm_pages=pages, hbm_budget_pages=pages,
                           host_pages=max(host_pages, slot), tiers=tiers,
                           kv=kv.view(torch.uint8).view(2 * layers, pages, page * heads * dim * 2))
        self.pool.import_placement(self.table, ctx)
        self.batch = KVBatch(self.pool, q_heads=heads * group, max_requests=max_requests or max(n, 1),
                             max_tokens=max_tokens or max(self.rows, 1), dtype=dtype, window=window, sinks=sinks)
        self.q = (sharp * torch.randn((self.rows, heads * group, dim), generator=self.gen, device="cuda")).to(dtype)

    def plan(self, **kw):
        self.batch.plan(self.sids, np.asarray(self.new, np.int32), num_tokens=self.rows, **kw)

    def close(self):
        self.pool.close()

    def seen(self, i):
        """[new, total] truth values of request i."""
        p = torch.arange(self.cached[i], self.total[i])[:, None]
        j = torch.arange(self.total[i])[None, :]
        s = j <= p
        if self.window:
            s &= (j > p - self.window) | (j < self.sinks)
        return s.cuda()

    def rows_of(self, i, kv, layer):
        """Request i's K or V, [total, heads, dim] in 64 bits; blocks that are nowhere in HBM: zeros."""
        t = self.total[i]
        j = torch.arange(t, device="cuda")
        page = torch.from_numpy(self.table[self.sids[i]].astype(np.int64)).cuda()[j // self.page]
        x = self.kv[2 * layer + kv][page.clamp(min=0), j % self.page].double()
        return torch.where((page >= 0)[:, None, None], x, torch.zeros_like(x))

    def attention64(self, layer, scale, q=None):
        """out, its bound's two magnitudes (|out| and the weighted |v|), lse and the largest
        sum of |q k| of a row, all in 64 bits."""
        Hq = self.heads * self.group
        q = (self.q if q is None else q).double()
        z = lambda *s: torch.zeros(s, dtype=torch.float64, device="cuda")
        out, mag, lse, dot = z(self.rows, Hq, self.dim), z(self.rows, Hq, self.dim), z(self.rows, Hq), z(self.rows, Hq)
        lse.fill_(-float("inf"))
        at = 0
        for i in range(self.n):
            m = self.new[i]
            if m == 0:
                continue
            k, v, hidden = self.rows_of(i, 0, layer), self.rows_of(i, 1, layer), ~self.seen(i)
            for h in range(Hq):
                kk, vv, x = k[:, h // self.group], v[:, h // self.group], q[at:at + m, h]
                s = (x @ kk.T) * scale
                s[hidden] = -float("inf")
                w = torch.softmax(s, 1)
                out[at:at + m, h] = w @ vv
                mag[at:at + m, h] = w @ vv.abs()
                lse[at:at + m, h] = torch.logsumexp(s, 1)
                dot[at:at + m, h] = (x.abs() @ kk.abs().T).masked_fill(hidden, 0).amax(1) * scale
            at += m
        return out, mag, lse, dot

    def check(self, got, lse, layer, scale, q=None):
        want, mag, want_lse, dot = self.attention64(layer, scale, q)
        u = UNIT[self.dtype]
        # a score is off by at most its magnitudes' sum times the accumulation's roundoff (head_dim
        # products added in 32 bits, with at most 2^-20 of the largest lost in all) and by the
        # rounding of its exponent; a weight by that much relatively, and by the type's roundoff; the
        # output by its own rounding
        score = dot * 2.0 ** -20 + 2.0 ** -19
        bound = u * want.abs() + (1.02 * u + 4 * score[..., None]) * mag + 1e-6
        err = (got.double() - want).abs()
        assert torch.isfinite(got).all()
        worst = (err / bound).max().item() if err.numel() else 0.0
        assert worst <= 1.0, worst
        if lse is not None:
            ends = torch.isinf(want_lse)
            assert torch.equal(torch.isinf(lse), ends)
            off = (lse.double() - want_lse).abs()[~ends]
            assert (off <= (4 * score[~ends] + 2.0 ** -18 * (1 + want_lse[~ends].abs()))).all(), off.max()
        return worst
