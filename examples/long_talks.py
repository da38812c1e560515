"""Talks of several sessions with one assistant, whose instructions all of them share, and which keep a part of
what was said:

    python examples/long_talks.py

The instructions are a session of their own, read once for all replies of a step (``KVBatch.plan`` with
``prefixes``).  Each step adds up the attention weights of the cached tokens (``KVBatch.add_weights``), and a
session that has grown past its limit keeps the heaviest half of its own tokens, in each layer and head
its own, besides the first and the last ones (``KVPool.evict_tokens``).

At the end every session's last hidden state is compared with that of a decoder that keeps everything.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import numpy as np
import torch

from voice_turns import Decoder


def run(sessions=5, steps=40, layers=3, instructions=333, limit=96, seed=0):
    """limit: tokens of its own that a session may hold; a step that passes it evicts down to half."""
    from paper_2606_22983_gb300.batch import KVBatch
    from paper_2606_22983_gb300.pool import KVPool
    kv_heads, group, dim, T = 2, 4, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    model = Decoder(layers, kv_heads, group, dim, 0, 0, seed)
    model.windowed = lambda layer: False
    most = limit + 8
    blocks = max(-(-instructions // T), -(-most // T)) + 1
    pages = -(-instructions // T) + sessions * (-(-most // T) + 1)
    shared = sessions                                    # the session that holds the instructions
    pool = KVPool(layers=layers, kv_heads=kv_heads, head_dim=dim, max_sessions=sessions + 1, max_blocks=blocks,
                  hbm_pages=pages, hbm_budget_pages=pages, host_pages=0)
    batch = KVBatch(pool, q_heads=kv_heads * group, max_requests=sessions, max_tokens=max(instructions, 8 * sessions),
                    prefix_rows=8 * sessions)
    weights = torch.zeros((layers, sessions + 1, kv_heads, blocks * T), device="cuda")
    heard = torch.randn((instructions, model.hidden), generator=gen, device="cuda").bfloat16()
    said = [heard] * sessions                            # what each session's rows see, with the instructions
    held, last, evicted = [0] * sessions, [None] * sessions, 0

    def forward(x):
        for layer in range(layers):
            q, k, v = model.project(layer, x)
            batch.write(layer, k, v)
            out, lse = batch.attention(layer, q, return_lse=True)
            batch.add_weights(layer, q, lse, weights[layer])
            x = x + out.reshape(len(x), -1) @ model.out[layer]
        return x

    try:
        pool.import_placement(np.full((sessions + 1, blocks), -1, np.int32), np.zeros(sessions + 1, np.int32))
        pool.append(shared, instructions)
        batch.plan(np.array([shared], np.int32), np.array([instructions], np.int32))
        forward(heard)
        sids = np.arange(sessions, dtype=np.int32)
        for _ in range(steps):
            lens = rng.integers(1, 8, sessions).astype(np.int32)
            over = np.array([s for s in range(sessions) if held[s] + lens[s] > limit], np.int32)
            if len(over):
                keeps = np.array([held[s] // 2 for s in over], np.int32)
                pool.evict_tokens(over, keeps, weights, first=2, last=8)
                evicted += int(sum(held[s] for s in over) - keeps.sum())
                for s, n in zip(over, keeps):
                    held[s] = int(n)
            for s in range(sessions):
                pool.append(s, int(lens[s]))
                held[s] += int(lens[s])
            x = torch.randn((int(lens.sum()), model.hidden), generator=gen, device="cuda").bfloat16()
            batch.plan(sids, lens, prefixes=np.full(sessions, shared, np.int32))
            y = forward(x)
            at = 0
            for s, n in enumerate(lens.tolist()):
                said[s] = torch.cat([said[s], x[at:at + n]])
                last[s] = y[at + n - 1]
                at += n
        pool.sync()
        apart = [((last[s].float() - (want := model.without_cache(said[s])[-1].float())).norm() / want.norm()).item()
                 for s in range(sessions)]
        return {"sessions": sessions, "said": [len(x) - instructions for x in said], "held": held, "evicted": evicted,
                "apart": max(apart)}
    finally:
        torch.cuda.synchronize()
        pool.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--sessions", type=int, default=5)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--limit", type=int, default=96)
    args = ap.parse_args()
    from paper_2606_22983_gb300 import build
    build()
    r = run(args.sessions, args.steps, limit=args.limit)
    print(f"{r['sessions']} sessions behind one prefix said {min(r['said'])} to {max(r['said'])} tokens and hold "
          f"{min(r['held'])} to {max(r['held'])}, {r['evicted']} evicted; last hidden states within {r['apart']:.1e} "
          f"of a decoder that keeps all")


if __name__ == "__main__":
    main()
