"""The performance cases of a serving step on the paged KV pool: what an engine calls between
one turn's ``lv_turn`` and the next, layer by layer.

  plan     a step's batch: block tables, rows, positions and the slot map of the new tokens
           from the requests' lengths (``KVBatch.plan``)
  write    the new tokens' K and V rows into their pages (``KVBatch.write``)
  attend   attention of each request's new tokens over its paged context (``KVBatch.attention``):
           single tokens, chunks, and both in one batch
  window   the same with a sliding window and a few first tokens that stay visible

With ``own`` false each runs in its plain form, in elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

# KV shapes of the pools: a two-layer model's, and the larger benchmark model's with fewer layers
TINY = dict(layers=2, kv_heads=2, head_dim=64, page_tokens=16)
THINKER = dict(layers=2, kv_heads=4, head_dim=128, page_tokens=16)
TABLES = dict(layers=1, kv_heads=1, head_dim=8, page_tokens=16)     # a plan reads tables, no KV

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
MOST_KV = 1 << 31          # bytes of K and V that a drawn case's step reads
MOST_PAIRS = 1 << 32       # query rows times keys of a drawn case (the largest listed: 8 * 32 * 4096^2)
MOST_ROWS = 16384          # new tokens of a drawn case


def _case(kind, name=None, **kw):
    """requests: sessions in the step, of ctx_lo..ctx_hi cached tokens; the first ``chunks`` of
    them bring chunk_lo..chunk_hi new tokens, each other one ``rest``; pad: rows of the step's
    tensors that no request owns.  ``lengths`` seeds the lengths (they belong to the case)."""
    c = dict(kind=kind, requests=1, ctx_lo=0, ctx_hi=0, chunks=0, chunk_lo=1, chunk_hi=1, rest=1, pad=0,
             q_heads=32, window=0, sinks=0, dtype="bf16", source="bf16", lse=False, lengths=1)
    c.update(THINKER)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step's plan: 64 running sessions, one new token each
        _case("plan", "plan_decode", requests=64, ctx_lo=2048, ctx_hi=16000, **TABLES),
        # as many sessions as the largest workload holds, chunks of speech and single tokens
        # mixed, some without new tokens, in a step padded to a fixed number of rows
        _case("plan", "plan_ragged", requests=1024, ctx_lo=256, ctx_hi=3500, chunks=96, chunk_lo=0, chunk_hi=129,
              pad=77, **TABLES),
        # the rows of a decode step: latency only
        _case("write", "write_decode", requests=64, ctx_lo=1, ctx_hi=4000, dtype="f16", source="f16"),
        # prompts' rows, rotated in 32 bits and rounded as they are stored
        _case("write", "write_prompts", requests=9, ctx_lo=0, ctx_hi=900, chunks=9, chunk_lo=1000, chunk_hi=2000,
              source="f32"),
        # the smallest call: one short session of the two-layer model
        _case("attend", "decode_one", requests=1, ctx_lo=77, ctx_hi=77, q_heads=4, **TINY),
        # a decode step of 61 sessions in a captured step of 64 rows
        _case("attend", "decode_many", requests=61, ctx_lo=2048, ctx_hi=16000, pad=3),
        # long voice sessions, single tokens
        _case("attend", "decode_long", requests=16, ctx_lo=32768, ctx_hi=65000, dtype="f16"),
        # the user's next utterance, 500 tokens, over one long context
        _case("attend", "chunk_long", requests=1, ctx_lo=64000, ctx_hi=64000, chunks=1, chunk_lo=500, chunk_hi=500),
        # chunks and single tokens in one step
        _case("attend", "mixed", requests=50, ctx_lo=700, ctx_hi=9000, chunks=3, chunk_lo=600, chunk_hi=1500,
              lse=True),
        # fresh prompts of one length: the largest
        _case("attend", "prompts", requests=8, ctx_lo=0, ctx_hi=0, chunks=8, chunk_lo=4096, chunk_hi=4096),
        # single tokens under a window of 4000 tokens and four first ones
        _case("window", "window_decode", requests=64, ctx_lo=1000, ctx_hi=30000, window=4000, sinks=4, lse=True),
        # chunks under a shorter window, the first 17 tokens visible
        _case("window", "window_chunk", requests=5, ctx_lo=100, ctx_hi=12000, chunks=5, chunk_lo=1500, chunk_hi=2100,
              window=1024, sinks=17, dtype="f16"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng: random.Random):
    kind = rng.choice(["plan", "write", "attend", "attend", "attend", "window", "window"])
    kv_heads = rng.choice([1, 2, 4, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    dim = rng.choice([64, 64, 96, 128, 128])
    shape = dict(kv_heads=kv_heads, q_heads=kv_heads * group, head_dim=dim,
                 page_tokens=rng.choice([16, 16, 16, 32, 64]), layers=rng.choice([1, 2, 3]))
    dtype = rng.choice(["bf16", "bf16", "f16"])
    lengths = rng.randrange(1 << 30)
    row = 4 * kv_heads * dim                       # bytes of one token's K and V in a layer
    if kind == "plan":
        requests = _log(rng, 1, 1024)
        shape.update(layers=1, kv_heads=1, q_heads=group, head_dim=8)
        return _case(kind, requests=requests, ctx_lo=1, ctx_hi=_log(rng, 16, min(60000, 4_000_000 // requests)),
                     chunks=rng.randint(0, requests), chunk_lo=0, chunk_hi=_log(rng, 1, max(1, 40000 // requests)),
                     rest=rng.choice([0, 1, 1, 3]), pad=rng.choice([1, 5, 100]), dtype=dtype, lengths=lengths, **shape)
    if kind == "write":
        requests = _log(rng, 1, 256)
        hi = _log(rng, 1, MOST_ROWS // requests)
        return _case(kind, requests=requests, ctx_lo=0, ctx_hi=_log(rng, 1, 3000), chunks=requests,
                     chunk_lo=max(1, hi // 3), chunk_hi=hi, pad=rng.choice([0, 0, 9]), dtype=dtype,
                     source=rng.choice([dtype, dtype, "f32"]), lengths=lengths, **shape)
    c = dict(dtype=dtype, lse=rng.random() < 0.3, lengths=lengths, **shape)
    if kind == "window":
        c.update(window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 4, 33, 130]))
    if rng.random() < 0.5:                         # single tokens, or a few (a draft to verify)
        requests = _log(rng, 1, 256)
        most = max(8, min(65000, MOST_KV // (row * requests)))
        hi = _log(rng, 8, most)
        return _case(kind, requests=requests, ctx_lo=max(1, hi // rng.choice([1, 3, 20])), ctx_hi=hi,
                     rest=rng.choice([1, 1, 1, 2, 4, 7]), **c)
    chunks = rng.choice([1, 1, 2, 3, 5, 12])
    requests = chunks + rng.choice([0, 0, 1, 20, 60])
    hi = _log(rng, 17, min(4096, MOST_ROWS // chunks))
    lo = max(1, hi // rng.choice([1, 2, 9]))
    # the chunks' query rows times the longest context they may have
    most = max(1, min(50000, MOST_KV // (row * requests), MOST_PAIRS // (chunks * hi * c["q_heads"]) - hi))
    ctx = _log(rng, 1, most)
    return _case(kind, requests=requests, ctx_lo=rng.choice([0, ctx // 4, ctx]) if requests == chunks else ctx // 4,
                 ctx_hi=ctx, chunks=chunks, chunk_lo=lo, chunk_hi=hi, **c)


# ------------------------------------------------------------------ lengths and work
def _lengths(c):
    """(cached tokens, new tokens) of every request."""
    rng = random.Random(c["lengths"])
    cached, new = [], []
    for i in range(c["requests"]):
        cached.append(_log(rng, c["ctx_lo"], c["ctx_hi"]) if c["ctx_hi"] > c["ctx_lo"] else c["ctx_lo"])
        new.append(rng.randint(c["chunk_lo"], c["chunk_hi"]) if i < c["chunks"] else c["rest"])
    return cached, new


def _seen(p, window, sinks):
    """Keys that a query at position p sees: itself and what precedes it in the window, and the sinks."""
    lo = max(0, p - window + 1) if window else 0
    return p + 1 - lo + min(sinks, lo)


def work(case):
    c = case
    cached, new = _lengths(c)
    T, H, D, Hq = c["page_tokens"], c["kv_heads"], c["head_dim"], c["q_heads"]
    rows = sum(new)
    if c["kind"] == "plan":
        blocks = sum((a + b + T - 1) // T for a, b in zip(cached, new))
        width = max((a + b + T - 1) // T for a, b in zip(cached, new))
        n = c["requests"]
        return {"bytes": 4 * blocks + 4 * n * width + 12 * (rows + c["pad"]) + 28 * n, "flops": 0}
    if c["kind"] == "write":
        src = 4 if c["source"] == "f32" else 2
        return {"bytes": rows * (2 * H * D * (src + 2) + 8), "flops": 0}
    pairs, keys = 0, 0
    for a, b in zip(cached, new):
        if b == 0:
            continue
        pairs += sum(_seen(p, c["window"], c["sinks"]) for p in range(a, a + b))
        lo = max(0, a - c["window"] + 1) if c["window"] else 0       # the first query's window start
        keys += a + b - lo + min(c["sinks"], lo)
    return {"bytes": keys * H * D * 4 + rows * Hq * D * 4 + (4 * rows * Hq if c["lse"] else 0),
            "flops": 4 * D * Hq * pairs}


# ------------------------------------------------------------------ state
class _State:
    pass


def _normal(shape, dtype, gen, std=1.0):
    """Normal values of a 16-bit type, made in pieces."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        x = flat[i:i + (1 << 28)]
        x.normal_(0.0, std, generator=gen)
    return out


def prepare(case, seed):
    c = case
    s = _State()
    s.case = c
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    T, H, D, L = c["page_tokens"], c["kv_heads"], c["head_dim"], c["layers"]
    dtype = DTYPES[c["dtype"]]
    cached, new = _lengths(c)
    n = c["requests"]
    s.new, s.total = new, [a + b for a, b in zip(cached, new)]
    s.rows = sum(new) + c["pad"]
    s.layer = L - 1
    # a pool with twice the step's sessions, their blocks scattered over its pages
    sessions = min(4096, 2 * n + 1)
    s.sids_list = rng.sample(range(sessions), n)
    blocks = [(x + T - 1) // T for x in s.total]
    width = max(max(blocks), 1)
    pages = sum(blocks) + 5
    s.kv = _normal((2 * L, pages, T, H, D), dtype, gen)
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((sessions, width), -1, dtype=torch.int32)
    ctx = torch.zeros(sessions, dtype=torch.int32)
    host, at = order.cpu(), 0
    for sid, b, x in zip(s.sids_list, blocks, s.total):
        table[sid, :b] = host[at:at + b]
        ctx[sid] = x
        at += b
    s.sids = torch.tensor(s.sids_list, dtype=torch.int32, device="cuda")
    s.lens = torch.tensor(new, dtype=torch.int32, device="cuda")
    s.longest = max(new)
    s.table, s.ctx = table.cuda(), ctx.cuda()
    s.K, s.V = s.kv[2 * s.layer], s.kv[2 * s.layer + 1]
    if c["kind"] == "write":
        # K and V as a fused projection leaves them: one row of both per token, V's heads after K's
        src = DTYPES[c["source"]]
        fused = torch.empty((s.rows, 2 * H, D), dtype=src, device="cuda").normal_(0.0, 1.0, generator=gen)
        s.k, s.v = fused[:, :H], fused[:, H:]
    elif c["kind"] in ("attend", "window"):
        s.q = _normal((s.rows, c["q_heads"], D), dtype, gen, 1.5)
        s.scale = D ** -0.5
    if own:
        from paper_2606_22983_gb300.batch import KVBatch
        from paper_2606_22983_gb300.pool import KVPool
        s.pool = KVPool(layers=L, kv_heads=H, head_dim=D, page_tokens=T, max_sessions=sessions, max_blocks=width,
                        hbm_pages=pages, hbm_budget_pages=pages, host_pages=0,
                        kv=s.kv.view(torch.uint8).view(2 * L, pages, T * H * D * 2))
        s.pool.import_placement(table.numpy(), ctx.numpy())
        s.batch = KVBatch(s.pool, q_heads=c["q_heads"], max_requests=n, max_tokens=max(s.rows, 1), dtype=dtype,
                          window=c["window"], sinks=c["sinks"])
        s.batch.plan(s.sids, s.lens, num_tokens=s.rows, max_len=s.longest)
        s.pool.sync()
    else:
        s.starts, s.kv_lens, s.tables, s.positions, s.slots = _plain_plan(s)
    return s


# ------------------------------------------------------------------ the plain forms
def _plain_plan(s):
    T = s.case["page_tokens"]
    sids, lens = s.sids.long(), s.lens.long()
    ends = lens.cumsum(0)
    starts = torch.cat([ends.new_zeros(1), ends])
    total = s.ctx[sids].long()
    blocks = (total + T - 1) // T
    tables = s.table[sids]
    at = torch.arange(tables.shape[1], device="cuda")
    tables = torch.where(at[None, :] < blocks[:, None], tables, torch.full_like(tables, -1))
    row = torch.arange(s.rows, device="cuda")
    live = row < ends[-1]
    req = torch.searchsorted(ends, row, right=True).clamp(max=len(s.new) - 1)
    pos = total[req] - lens[req] + row - starts[req]
    pos = torch.where(live, pos, torch.zeros_like(pos))
    slots = tables[req, pos // T].long() * T + pos % T
    none = torch.full_like(pos, -1)
    return (starts.to(torch.int32), total.to(torch.int32), tables, torch.where(live, pos, none).to(torch.int32),
            torch.where(live, slots, none))


def _plain_write(s):
    H, D = s.case["kv_heads"], s.case["head_dim"]
    n = sum(s.new)
    at = s.slots[:n]
    s.K.view(-1, H, D)[at] = s.k[:n].to(s.K.dtype)
    s.V.view(-1, H, D)[at] = s.v[:n].to(s.V.dtype)
    return s.K, s.V


def _visible(c, first, count, keys, kdev):
    """[count, keys]: which keys the queries at first..first+count see."""
    p = torch.arange(first, first + count, device=kdev)[:, None]
    j = torch.arange(keys, device=kdev)[None, :]
    seen = j <= p
    if c["window"]:
        seen = seen & ((j > p - c["window"]) | (j < c["sinks"]))
    return seen


def _plain_attention(s):
    c = s.case
    H, D, Hq, T = c["kv_heads"], c["head_dim"], c["q_heads"], c["page_tokens"]
    G = Hq // H
    out = torch.zeros((s.rows, Hq, D), dtype=torch.float32, device="cuda")
    lse = torch.full((s.rows, Hq), -math.inf, dtype=torch.float32, device="cuda") if c["lse"] else None
    at = 0
    for i, (m, total) in enumerate(zip(s.new, s.total)):
        if m == 0:
            continue
        pages = s.tables[i, :(total + T - 1) // T].long()
        k = s.K[pages].view(-1, H, D)[:total].float().permute(1, 2, 0)                 # [H, D, keys]
        v = s.V[pages].view(-1, H, D)[:total].float().permute(1, 0, 2)                 # [H, keys, D]
        q = s.q[at:at + m].float().view(m, H, G, D).permute(1, 2, 0, 3).reshape(H, G * m, D)
        score = torch.matmul(q, k).view(H, G, m, total) * s.scale
        score = score.masked_fill(~_visible(c, total - m, m, total, "cuda"), -math.inf)
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        del score
        norm = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(H, G * m, total), v).view(H, G, m, D) / norm
        out[at:at + m] = o.permute(2, 0, 1, 3).reshape(m, Hq, D)
        if lse is not None:
            lse[at:at + m] = (top + norm.log()).view(H, G, m).permute(2, 0, 1).reshape(m, Hq)
        at += m
    out = out.to(s.q.dtype)
    return (out, lse) if lse is not None else out


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    kind = s.case["kind"]
    if not own:
        return _plain_plan(s) if kind == "plan" else _plain_write(s) if kind == "write" else _plain_attention(s)
    if kind == "plan":
        b = s.batch
        b.plan(s.sids, s.lens, num_tokens=s.rows, max_len=s.longest)
        n = len(s.new)
        return b.row_starts[:n + 1], b.kv_lens[:n], b.tables[:n], b.positions[:s.rows], b.slots[:s.rows]
    if kind == "write":
        s.batch.write(s.layer, s.k, s.v)
        return s.K, s.V
    if s.case["lse"]:
        return s.batch.attention(s.layer, s.q, scale=s.scale, return_lse=True)
    return s.batch.attention(s.layer, s.q, scale=s.scale)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """The written rows, or the attention, in 64 bits: request by request and head by head,
    from the block tables as they were made."""
    c = case
    if c["kind"] == "plan":
        return None
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    T, H, D, Hq = c["page_tokens"], c["kv_heads"], c["head_dim"], c["q_heads"]
    if c["kind"] == "write":
        if s.K.numel() > 1 << 28:
            return None
        K, V = s.K.double().view(-1, H, D), s.V.double().view(-1, H, D)
        at = 0
        for sid, m, total in zip(s.sids_list, s.new, s.total):
            for t in range(m):
                block, off = divmod(total - m + t, T)
                slot = int(s.table[sid, block]) * T + off if t == 0 or off == 0 else slot + 1
                K[slot], V[slot] = s.k[at + t].double(), s.v[at + t].double()
            at += m
        return K.view(s.K.shape), V.view(s.V.shape)
    if 4 * D * sum(m * total for m, total in zip(s.new, s.total)) * Hq > 4e12:
        return None
    out = torch.zeros((s.rows, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((s.rows, Hq), -math.inf, dtype=torch.float64, device="cuda") if c["lse"] else None
    at = 0
    for sid, m, total in zip(s.sids_list, s.new, s.total):
        pages = s.table[sid].long()
        token = torch.arange(total, device="cuda")
        page, off = pages[token // T], token % T
        step = max(1, (1 << 27) // max(total, 1))
        for h in range(H if m else 0):
            k, v = s.K[page, off, h].double(), s.V[page, off, h].double()
            heads = range(h * (Hq // H), (h + 1) * (Hq // H))
            for a in range(0, m, step):
                b = min(m, a + step)
                hidden = ~_visible(c, total - m + a, b - a, total, "cuda")
                for g in heads:
                    x = (s.q[at + a:at + b, g].double() @ k.T) * s.scale
                    x[hidden] = -math.inf
                    z = torch.logsumexp(x, 1)
                    out[at + a:at + b, g] = torch.exp(x - z[:, None]) @ v
                    if lse is not None:
                        lse[at + a:at + b, g] = z
        at += m
    return (out, lse) if lse is not None else out
