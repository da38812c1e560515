"""A pool with weights of its sessions' tokens, and the choice and the moves by their definitions on the host."""
import math

import numpy as np
import torch


class Kept:
    """Sessions of ``total`` tokens over scattered pages, K and V by a counter (every row its own bytes)."""

    def __init__(self, total, *, layers=2, heads=2, dim=64, page=16, elem=2, spare=3, seed=0, host=(), tiers=0,
                 room=0, stream=None, slack=0):
        from paper_2606_22983_gb300.pool import KVPool
        rng = np.random.default_rng(seed)
        self.rng, self.total, self.page, self.layers, self.heads = rng, list(total), page, layers, heads
        n = len(total)
        sessions = 2 * n + 1
        self.sids = rng.permutation(sessions)[:n].astype(np.int32)
        blocks = [-(-t // page) for t in total]
        width = max(blocks + [1]) + 1
        pages = max(sum(blocks) + spare, 1)
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((sessions, width), -1, np.int32)
        self.ctx = np.zeros(sessions, np.int32)
        at = slot = 0
        for i, (sid, b, t) in enumerate(zip(self.sids, blocks, total)):
            self.table[sid, :b] = order[at:at + b]
            self.ctx[sid] = t
            for blk in range(b):
                if (i, blk) in host:
                    self.table[sid, blk] = -2 - slot
                    slot += 1
            at += b
        self.kv = torch.from_numpy(rng.integers(0, 256, (2 * layers, pages, page, heads, dim * elem), dtype=np.uint8)).cuda()
        self.pool = KVPool(layers=layers, kv_heads=heads, head_dim=dim, page_tokens=page, elem_bytes=elem,
                           max_sessions=sessions, max_blocks=width, hbm_pages=pages, hbm_budget_pages=pages,
                           host_pages=max(room, slot), tiers=tiers, stream=stream,
                           kv=self.kv.view(2 * layers, pages, page * heads * dim * elem))
        self.pool.import_placement(self.table, self.ctx)
        self.tokens = width * page + slack
        self.weights = torch.from_numpy(self.some_weights((layers, sessions, heads, self.tokens))).cuda()

    def some_weights(self, shape):
        """Few different values, so that many are equal, and a quarter zeros of either sign."""
        x = np.exp(self.rng.normal(-3, 2, shape)).astype(np.float32).round(2)
        zero = self.rng.random(shape)
        x[zero < 0.25] = 0.0
        x[zero < 0.1] = -0.0
        return x

    def close(self):
        self.pool.close()

    def choose(self, i, keep, first, last):
        """[layers, heads, keep]: request i's kept tokens by the definition."""
        c = self.total[i]
        keep = min(keep, c)
        first = min(first, keep)
        last = min(last, keep - first)
        out = np.zeros((self.layers, self.heads, keep), np.int32)
        w = self.weights.cpu().numpy()
        for layer in range(self.layers):
            for h in range(self.heads):
                x = w[layer, self.sids[i], h]
                rank = lambda j: math.inf if math.isnan(x[j]) else x[j]       # (a NaN above infinity)
                order = sorted(range(first, c - last), key=lambda j: (not math.isnan(x[j]), -rank(j), j))
                chosen = list(range(first)) + order[:keep - first - last] + list(range(c - last, c))
                out[layer, h] = sorted(chosen)
        return out

    def moved(self, requests, keeps, kept, weights=True):
        """K, V and the weights after the requests' moves."""
        kv, w = self.kv.cpu().numpy().copy(), self.weights.cpu().numpy().copy()
        T = self.page
        for i, keep in zip(requests, keeps):
            c, sid = self.total[i], self.sids[i]
            if keep >= c:
                continue
            row = self.table[sid]
            place = lambda j: (row[j // T], j % T)
            for layer in range(self.layers):
                for h in range(self.heads):
                    x = kept[i][layer, h]
                    for j in range(2 * layer, 2 * layer + 2):
                        old = [kv[j][place(t)][h].copy() for t in x[:keep]]
                        for t in range(keep):
                            kv[j][place(t)][h] = old[t]
                    if weights:
                        old = w[layer, sid, h][x[:keep]].copy()
                        w[layer, sid, h, :c] = 0
                        w[layer, sid, h, :keep] = old
        return kv, w
