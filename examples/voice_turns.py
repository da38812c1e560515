"""Turns of a voice model's sessions, from the user's words to the reply, over a KV pool too small
for all of them:

    python examples/voice_turns.py

Each turn of a session is one ``lv_turn`` (its offloaded KV is loaded, other sessions' KV makes room,
its context grows by the user's tokens), then one step over the user's chunk, then steps of single
tokens for the reply, in which the other replying sessions take part.  A step plans its batch once and
runs every layer of a small attention-only decoder through ``KVBatch.write`` and ``KVBatch.attention``.
Layers alternate between full attention and a sliding window with first tokens that stay visible.

At the end every session's last hidden state is computed again without a cache, and compared.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch


class Decoder:
    """x <- x + attention(norm(x)) Wo, layer by layer; no positions but the mask's."""

    def __init__(self, layers, kv_heads, group, dim, window, sinks, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.layers, self.kv_heads, self.group, self.dim = layers, kv_heads, group, dim
        self.hidden, self.window, self.sinks = kv_heads * group * dim, window, sinks
        make = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float32) / math.sqrt(s[-2])
        self.qkv = make(layers, self.hidden, (group + 2) * kv_heads * dim).bfloat16()
        self.out = (make(layers, self.hidden, self.hidden) * 0.5).bfloat16()

    def windowed(self, layer):
        return layer % 2 == 1

    def project(self, layer, x):
        """Queries, keys and values of rows x: views of one projection."""
        y = torch.nn.functional.rms_norm(x, (self.hidden,)) @ self.qkv[layer]
        y = y.view(len(x), -1, self.dim)
        q = self.kv_heads * self.group
        return y[:, :q], y[:, q:q + self.kv_heads], y[:, q + self.kv_heads:]

    def step(self, batches, x):
        """Rows x of a planned step through every layer; batches: full attention's and the window's."""
        for layer in range(self.layers):
            q, k, v = self.project(layer, x)
            b = batches[self.windowed(layer)]
            b.write(layer, k, v)
            x = x + b.attention(layer, q).reshape(len(x), -1) @ self.out[layer]
        return x

    def without_cache(self, x):
        n = len(x)
        p, j = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None]
        for layer in range(self.layers):
            q, k, v = (y.transpose(0, 1).float() for y in self.project(layer, x))
            k, v = (y.repeat_interleave(self.group, 0) for y in (k, v))
            seen = j <= p
            if self.windowed(layer):
                seen &= (j > p - self.window) | (j < self.sinks)
            w = torch.softmax((q @ k.transpose(1, 2) / math.sqrt(self.dim)).masked_fill(~seen, -math.inf), -1)
            x = x + (w @ v).transpose(0, 1).reshape(n, -1).to(x.dtype) @ self.out[layer]
        return x


def run(sessions=6, turns=4, layers=4, seed=0):
    from paper_2606_22983_gb300 import lv
    from paper_2606_22983_gb300.batch import KVBatch
    from paper_2606_22983_gb300.pool import KVPool
    kv_heads, group, dim, T = 2, 4, 64, 16
    window, sinks = 96, 4
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    model = Decoder(layers, kv_heads, group, dim, window, sinks, seed)
    words = rng.integers(20, 150, (turns, sessions))
    replies = rng.integers(5, 30, turns)
    blocks = -(-int(words.sum(0).max() + sessions * replies.sum()) // T) + 1
    # about half of what the sessions come to hold (each replies in its own turn and in the next one)
    budget = int(sum(-(-int(words[:, s].sum() + 2 * replies.sum()) // T) for s in range(sessions)) * 0.55)
    pool = KVPool(layers=layers, kv_heads=kv_heads, head_dim=dim, max_sessions=sessions, max_blocks=blocks,
                  hbm_pages=budget, hbm_budget_pages=budget, host_pages=sessions * blocks)
    batches = [KVBatch(pool, q_heads=kv_heads * group, max_requests=sessions, max_tokens=256, **kw)
               for kw in ({}, dict(window=window, sinks=sinks))]
    # what each session was told and has said, as the embeddings a model would look up
    spoken = [torch.zeros((0, model.hidden), dtype=torch.bfloat16, device="cuda") for _ in range(sessions)]
    last = [None] * sessions
    now = 0

    def step(sids, lens):
        x = torch.randn((sum(lens), model.hidden), generator=gen, device="cuda").bfloat16()
        for b in batches:
            b.plan(np.array(sids, np.int32), np.array(lens, np.int32))
        y = model.step(batches, x)
        at = 0
        for sid, n in zip(sids, lens):
            spoken[sid] = torch.cat([spoken[sid], x[at:at + n]])
            last[sid] = y[at + n - 1]
            at += n

    try:
        for turn in range(turns):
            talking = []                            # sessions whose KV is resident and whose reply runs
            for sid in rng.permutation(sessions).tolist():
                now += 400_000
                lv.lv_turn(pool.handle, sid, now, int(words[turn, sid]), 2_000_000, 25, stream=pool.stream)
                step([sid], [int(words[turn, sid])])
                talking = (talking + [sid])[-2:]
                for _ in range(int(replies[turn])):
                    for s in talking:
                        pool.events(np.array([(lv.LV_EV_TURN_BEGIN, s, now, 0, 0)], lv.EVENT_DTYPE))
                        lv.lv_make_resident(pool.handle, s, now, 1, 0, -1, None, None, None, None, None, None,
                                            pool.stream)
                    step(talking, [1] * len(talking))
                for s in talking:
                    pool.events(np.array([(lv.LV_EV_TURN_END, s, now, 2_000_000, 25)], lv.EVENT_DTYPE))
        pool.sync()
        worst = 0.0
        for sid in range(sessions):
            want = model.without_cache(spoken[sid])[-1].float()
            worst = max(worst, ((last[sid].float() - want).norm() / want.norm()).item())
        st = pool.stats()
        return {"sessions": sessions, "turns": turns * sessions, "longest_context": max(len(x) for x in spoken),
                "pages_out": st["pages_out"], "pages_in": st["pages_in"], "error": worst}
    finally:
        torch.cuda.synchronize()
        pool.close()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--sessions", type=int, default=6)
    ap.add_argument("--turns", type=int, default=4)
    args = ap.parse_args()
    from paper_2606_22983_gb300 import build
    build()
    r = run(args.sessions, args.turns)
    print(f"{r['turns']} turns of {r['sessions']} sessions, contexts up to {r['longest_context']} tokens: "
          f"{r['pages_out']} pages moved out, {r['pages_in']} in; last hidden states within "
          f"{r['error']:.1e} of a run without a cache")


if __name__ == "__main__":
    main()
