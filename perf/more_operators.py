"""The performance cases of long and shared contexts on the paged KV pool:

  shared   attention of a step whose requests continue a prefix that another session holds, read
           once for all of them (``KVBatch.plan`` with ``prefixes``, ``KVBatch.attention``)
  weights  the attention weights that the cached tokens got from a step's rows, added up for
           every token and KV head (``KVBatch.add_weights``)
  select   the tokens of each session, layer and KV head to keep: the first and last ones, and
           those of the largest weight (``KVPool.select_kept``)
  compact  the kept tokens' K, V and weights to the front of their sessions' pages
           (``KVPool.compact``)

With ``own`` false each runs in its plain form, in elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

# KV shapes of the pools: a two-layer model's, and the larger benchmark model's with fewer layers
TINY = dict(layers=2, kv_heads=2, head_dim=64, page_tokens=16)
THINKER = dict(layers=2, kv_heads=4, head_dim=128, page_tokens=16)

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
MOST_KV = 1 << 30          # bytes of K and V that a drawn case's step reads, or moves
MOST_PAIRS = 1 << 29       # query rows times keys of a drawn case
MOST_ROWS = 8192           # new tokens of a drawn case


def _case(kind, name=None, **kw):
    """requests: sessions, of ctx_lo..ctx_hi cached tokens of their own.  Steps: the first ``chunks``
    requests bring chunk_lo..chunk_hi new tokens, each other one ``rest``; the requests continue
    ``prefixes`` shared ones of prefix_lo..prefix_hi tokens, each as many requests as the next (the
    last ``alone`` requests none); last: rows of a request that count (0: all).  select and compact:
    1 / ``keep`` of the context stays.  ``lengths`` seeds the lengths (they belong to the case)."""
    c = dict(kind=kind, requests=1, ctx_lo=0, ctx_hi=0, chunks=0, chunk_lo=1, chunk_hi=1, rest=1, q_heads=32,
             prefixes=0, prefix_lo=0, prefix_hi=0, alone=0, last=0, keep=2.0, first=0, recent=0, dtype="bf16",
             lse=False, lengths=1)
    c.update(THINKER)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: two sessions of the two-layer model behind a short greeting
        _case("shared", "shared_two", requests=2, ctx_lo=20, ctx_hi=60, prefixes=1, prefix_lo=77, prefix_hi=77,
              q_heads=4, **TINY),
        # a decode step of 64 sessions of one assistant: its instructions and tools in front of short talks
        _case("shared", "shared_decode", requests=64, ctx_lo=200, ctx_hi=2500, prefixes=1, prefix_lo=8192,
              prefix_hi=8192),
        # drafts of four tokens behind three assistants' prefixes of odd lengths, and sessions without one
        _case("shared", "shared_drafts", requests=43, ctx_lo=100, ctx_hi=4000, rest=4, prefixes=3, prefix_lo=1500,
              prefix_hi=12000, alone=4, dtype="f16", lse=True),
        # the sessions' first utterances, prefilled together behind the prefix
        _case("shared", "shared_chunks", requests=8, ctx_lo=0, ctx_hi=900, chunks=8, chunk_lo=200, chunk_hi=700,
              prefixes=1, prefix_lo=6000, prefix_hi=6000),
        # the smallest: one token's weights over one short session
        _case("weights", "weights_one", requests=1, ctx_lo=77, ctx_hi=77, q_heads=4, **TINY),
        # a decode step's weights
        _case("weights", "weights_decode", requests=61, ctx_lo=2048, ctx_hi=16000),
        # a long utterance's last 32 tokens decide what of the context before them is kept
        _case("weights", "weights_tail", requests=5, ctx_lo=20000, ctx_hi=60000, chunks=5, chunk_lo=100, chunk_hi=400,
              last=32, dtype="f16"),
        # whole prompts: the largest
        _case("weights", "weights_prompts", requests=4, chunks=4, chunk_lo=4096, chunk_hi=4096),
        # one short session of the two-layer model
        _case("select", "select_one", requests=1, ctx_lo=500, ctx_hi=500, first=4, recent=32, **TINY),
        # long sessions of the whole model cut to a quarter
        _case("select", "select_long", requests=12, ctx_lo=4000, ctx_hi=30000, keep=4.0, first=4, recent=128,
              **dict(THINKER, layers=48)),
        # the same two with their K and V moved
        _case("compact", "compact_one", requests=1, ctx_lo=500, ctx_hi=500, first=4, recent=32, **TINY),
        _case("compact", "compact_long", requests=4, ctx_lo=6000, ctx_hi=14000, keep=4.0, first=4, recent=128,
              **dict(THINKER, layers=48)),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 1)), math.log(max(hi, 1))))))))


def draw(rng: random.Random):
    kind = rng.choice(["shared", "shared", "shared", "weights", "weights", "select", "compact"])
    kv_heads = rng.choice([1, 2, 4, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
    dim = rng.choice([64, 64, 96, 128, 128])
    shape = dict(kv_heads=kv_heads, q_heads=kv_heads * group, head_dim=dim,
                 page_tokens=rng.choice([16, 16, 16, 32, 64]), layers=rng.choice([1, 2, 3]))
    c = dict(dtype=rng.choice(["bf16", "bf16", "f16"]), lengths=rng.randrange(1 << 30), **shape)
    row = 4 * kv_heads * dim                       # bytes of one token's K and V in a layer
    if kind in ("select", "compact"):
        c["layers"] = rng.choice([1, 2, 8, 31, 48])
        c["q_heads"] = kv_heads
        requests = _log(rng, 1, 64)
        most = (1 << 24) // (kv_heads * c["layers"]) if kind == "select" else MOST_KV // (row * c["layers"])
        hi = _log(rng, 100, max(100, min(60000, most // requests)))
        lo = max(100, hi // rng.choice([1, 3, 20]))
        # (so few first and last ones that some of the others stay in the shortest session too)
        return _case(kind, requests=requests, ctx_lo=lo, ctx_hi=hi, keep=rng.choice([1.3, 2.0, 4.0, 8.0]),
                     first=min(lo // 20, rng.choice([0, 1, 4, 33])),
                     recent=min(lo // 20, rng.choice([0, 1, 32, 128, 700])), **c)
    if kind == "shared":
        c["lse"] = rng.random() < 0.3
        prefix = _log(rng, 16, 30000)
        if rng.random() < 0.5:                     # single tokens, or a few (a draft to verify)
            requests = _log(rng, 1, 256)
            groups = rng.choice([1, 1, 2, min(5, requests)])
            hi = _log(rng, 8, max(8, min(20000, MOST_KV // (row * requests))))
            return _case(kind, requests=requests, ctx_lo=max(1, hi // rng.choice([1, 3, 20])), ctx_hi=hi,
                         rest=rng.choice([1, 1, 1, 2, 4, 7]), prefixes=min(groups, requests), prefix_lo=max(1, prefix // 3),
                         prefix_hi=prefix, alone=rng.choice([0, 0, requests // 3]), **c)
        chunks = rng.choice([1, 2, 3, 5, 12])
        requests = chunks + rng.choice([0, 0, 1, 20])
        hi = _log(rng, 17, min(2048, MOST_ROWS // chunks, int((MOST_PAIRS / (chunks * c["q_heads"])) ** 0.5)))
        keys = MOST_PAIRS // (chunks * hi * c["q_heads"])
        prefix = max(16, min(prefix, keys - hi))
        return _case(kind, requests=requests, ctx_lo=0, chunks=chunks,
                     ctx_hi=_log(rng, 1, max(1, min(3000, keys - hi - prefix))),
                     chunk_lo=max(1, hi // rng.choice([1, 2, 9])), chunk_hi=hi, prefixes=rng.choice([1, 1, 2]) if requests > 1 else 1,
                     prefix_lo=max(1, prefix // 2), prefix_hi=prefix, **c)
    if rng.random() < 0.5:
        requests = _log(rng, 1, 256)
        hi = _log(rng, 8, max(8, min(65000, MOST_KV // (row * requests))))
        return _case(kind, requests=requests, ctx_lo=max(1, hi // rng.choice([1, 3, 20])), ctx_hi=hi,
                     rest=rng.choice([1, 1, 1, 2, 4]), prefixes=rng.choice([0, 0, 1]), prefix_lo=33, prefix_hi=9000, **c)
    chunks = rng.choice([1, 1, 2, 3, 5])
    requests = chunks + rng.choice([0, 0, 1, 20])
    hi = _log(rng, 17, min(4096, MOST_ROWS // chunks, int((2 * MOST_PAIRS / (chunks * c["q_heads"])) ** 0.5)))
    last = rng.choice([0, 0, 16, 64])
    most = max(1, min(50000, MOST_KV // (row * requests), MOST_PAIRS // (chunks * (last or hi) * c["q_heads"]) - hi))
    ctx = _log(rng, 1, most)
    return _case(kind, requests=requests, ctx_lo=ctx // rng.choice([1, 4]), ctx_hi=ctx, chunks=chunks,
                 chunk_lo=max(1, hi // rng.choice([1, 2, 9])), chunk_hi=hi, last=last, **c)


# ------------------------------------------------------------------ lengths and work
def _lengths(c):
    """(cached tokens, new tokens, prefix's number or -1) of every request; tokens of the prefixes."""
    rng = random.Random(c["lengths"])
    cached, new, of = [], [], []
    n, shared = c["requests"], c["requests"] - c["alone"]
    for i in range(n):
        cached.append(_log(rng, c["ctx_lo"], c["ctx_hi"]) if c["ctx_hi"] > c["ctx_lo"] else c["ctx_lo"])
        new.append(rng.randint(c["chunk_lo"], c["chunk_hi"]) if i < c["chunks"] else c["rest"])
        of.append(i * c["prefixes"] // shared if c["prefixes"] and i < shared else -1)
    prefix = [rng.randint(c["prefix_lo"], c["prefix_hi"]) for _ in range(c["prefixes"])]
    if c["kind"] in ("select", "compact"):
        new = [0] * n
    return cached, new, of, prefix


def _keeps(c, cached):
    """Tokens that each session keeps."""
    return [min(x, max(c["first"] + c["recent"], int(x / c["keep"]))) for x in cached]


def work(case):
    c = case
    cached, new, of, prefix = _lengths(c)
    L, H, D, Hq = c["layers"], c["kv_heads"], c["head_dim"], c["q_heads"]
    rows = sum(new)
    if c["kind"] == "select":
        return {"bytes": 4 * L * H * (sum(cached) + sum(_keeps(c, cached))), "flops": 0}
    if c["kind"] == "compact":
        # K and V of the kept tokens read and written, their places and their weights with them,
        # and the weights behind them cleared
        kept = sum(_keeps(c, cached))
        return {"bytes": L * H * (kept * (2 * D * 2 * 2 + 4 + 4) + 4 * sum(cached)), "flops": 0}
    if c["kind"] == "shared":
        pairs = sum(m * (a + (prefix[p] if p >= 0 else 0)) + m * (m + 1) // 2 for a, m, p in zip(cached, new, of))
        keys = sum(a + m for a, m in zip(cached, new)) + sum(prefix)
        return {"bytes": keys * H * D * 4 + rows * Hq * D * 4 + (4 * rows * Hq if c["lse"] else 0),
                "flops": 4 * D * Hq * pairs}
    keys = sum(a + m for a, m in zip(cached, new)) + sum(prefix)
    pairs = counted = 0
    for a, m, p in zip(cached, new, of):
        n = min(m, c["last"]) if c["last"] else m
        pairs += n * (a + m - n + (prefix[p] if p >= 0 else 0)) + n * (n + 1) // 2
        counted += n
    return {"bytes": keys * H * (2 * D + 8) + counted * Hq * (2 * D + 4), "flops": 2 * D * Hq * pairs}


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
    cached, new, of, prefix = _lengths(c)
    n = c["requests"]
    s.new, s.total, s.prefix = new, [a + b for a, b in zip(cached, new)], prefix
    s.of = of
    s.rows = sum(new)
    s.layer = L - 1
    # a pool with some more sessions than the step's and the prefixes', their blocks scattered over its pages
    held = s.total + prefix
    sessions = min(4096, len(held) + 3)
    ids = rng.sample(range(sessions), len(held))
    s.sids_list, s.prefix_sids = ids[:n], ids[n:]
    blocks = [(x + T - 1) // T for x in held]
    width = max(max(blocks), 1)
    pages = sum(blocks) + 5
    # (choosing tokens reads no K and V: its pool has one layer's pages for all)
    s.kv = _normal((2 if c["kind"] == "select" else 2 * L, pages, T, H, D), dtype, gen)
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((sessions, width), -1, dtype=torch.int32)
    ctx = torch.zeros(sessions, dtype=torch.int32)
    host, at = order.cpu(), 0
    for sid, b, x in zip(ids, blocks, held):
        table[sid, :b] = host[at:at + b]
        ctx[sid] = x
        at += b
    s.table = table.cuda()
    s.tokens = width * T
    s.sids = torch.tensor(s.sids_list, dtype=torch.int32, device="cuda")
    if c["kind"] in ("select", "compact"):
        # what decode steps leave: a few tokens have most, many next to nothing, and some the same
        s.weights = torch.empty((L, sessions, H, s.tokens), dtype=torch.float32, device="cuda")
        s.weights.normal_(-6.0, 3.0, generator=gen).exp_()
        s.weights[s.weights < 2e-4] = 0.0
        s.keeps = _keeps(c, cached)
        s.keeps_dev = torch.tensor(s.keeps, dtype=torch.int32, device="cuda")
        s.most = max(s.keeps)
    else:
        s.q = _normal((s.rows, c["q_heads"], D), dtype, gen, 1.5)
        s.scale = D ** -0.5
    if c["kind"] == "compact":
        s.kept = _plain_select(s)
    if c["kind"] == "weights":
        s.weights = torch.empty((L, sessions, H, s.tokens), dtype=torch.float32, device="cuda")
        s.weights.normal_(-8.0, 1.5, generator=gen).exp_()      # a few steps' weights
        s.lse = torch.empty((s.rows, c["q_heads"]), dtype=torch.float32, device="cuda")
        _plain_rows(s, lambda i, r0, r1, score, v, k0: s.lse[r0:r1].copy_(
            torch.logsumexp(score, 3).permute(2, 0, 1).reshape(r1 - r0, -1)))
    if own:
        from paper_2606_22983_gb300.batch import KVBatch
        from paper_2606_22983_gb300.pool import KVPool
        J = 2 * L
        bytes_of = s.kv.view(torch.uint8).view(s.kv.shape[0], pages, T * H * D * 2)
        s.pool = KVPool(layers=L, kv_heads=H, head_dim=D, page_tokens=T, max_sessions=sessions, max_blocks=width,
                        hbm_pages=pages, hbm_budget_pages=pages, host_pages=0,
                        kv=[bytes_of[j % s.kv.shape[0]] for j in range(J)])
        s.pool.import_placement(table.numpy(), ctx.numpy())
        if c["kind"] in ("shared", "weights"):
            s.batch = KVBatch(s.pool, q_heads=c["q_heads"], max_requests=n, max_tokens=max(s.rows, 1), dtype=dtype,
                              prefix_rows=s.rows if prefix else 0)
            more = {}
            if prefix:
                more["prefixes"] = torch.tensor([s.prefix_sids[p] if p >= 0 else -1 for p in of], dtype=torch.int32,
                                                device="cuda")
            lens = torch.tensor(new, dtype=torch.int32, device="cuda")
            s.batch.plan(s.sids, lens, num_tokens=s.rows, max_len=max(new), **more)
        s.pool.sync()
    return s


# ------------------------------------------------------------------ the plain forms
def _keys_of(s, kv, sid, total):
    """K or V of a session, [total, H, D] in 32 bits."""
    c = s.case
    pages = s.table[sid, :(total + c["page_tokens"] - 1) // c["page_tokens"]].long()
    return s.kv[2 * s.layer + kv][pages].view(-1, c["kv_heads"], c["head_dim"])[:total].float()


def _plain_rows(s, take):
    """take(request, first row, end, scores [H, G, rows, keys], V [keys, H, D], keys before its own) of
    every request's counted rows: the prefix's keys first, then its own."""
    c = s.case
    H, D, Hq = c["kv_heads"], c["head_dim"], c["q_heads"]
    G = Hq // H
    want_v = c["kind"] == "shared"
    at = 0
    for i, (m, total) in enumerate(zip(s.new, s.total)):
        own_k = _keys_of(s, 0, s.sids_list[i], total)
        own_v = _keys_of(s, 1, s.sids_list[i], total) if want_v else None
        before = 0
        if s.of[i] >= 0:
            before = s.prefix[s.of[i]]
            sid = s.prefix_sids[s.of[i]]
            own_k = torch.cat([_keys_of(s, 0, sid, before), own_k])
            own_v = torch.cat([_keys_of(s, 1, sid, before), own_v]) if want_v else None
        k = own_k.permute(1, 2, 0)                                                     # [H, D, keys]
        keys = before + total
        skip = max(0, m - c["last"]) if c["last"] else 0
        step = max(1, (1 << 29) // max(1, Hq * keys))      # rows whose scores are held at once
        for a in range(skip, m, step):
            b = min(m, a + step)
            q = s.q[at + a:at + b].float().view(b - a, H, G, D).permute(1, 2, 0, 3).reshape(H, G * (b - a), D)
            score = torch.matmul(q, k).view(H, G, b - a, keys) * s.scale
            p = torch.arange(keys - m + a, keys - m + b, device="cuda")[:, None]
            score = score.masked_fill(torch.arange(keys, device="cuda")[None, :] > p, -math.inf)
            take(i, at + a, at + b, score, own_v, before)
        at += m


def _plain_shared(s):
    c = s.case
    H, D, Hq = c["kv_heads"], c["head_dim"], c["q_heads"]
    G = Hq // H
    out = torch.zeros((s.rows, Hq, D), dtype=torch.float32, device="cuda")
    lse = torch.empty((s.rows, Hq), dtype=torch.float32, device="cuda")

    def take(i, r0, r1, score, v, before):
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        norm = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(H, G * (r1 - r0), -1), v.permute(1, 0, 2)).view(H, G, r1 - r0, D) / norm
        out[r0:r1] = o.permute(2, 0, 1, 3).reshape(r1 - r0, Hq, D)
        lse[r0:r1] = (top + norm.log()).view(H, G, r1 - r0).permute(2, 0, 1).reshape(r1 - r0, Hq)

    _plain_rows(s, take)
    out = out.to(s.q.dtype)
    return (out, lse) if c["lse"] else out


def _plain_weights(s):
    H = s.case["kv_heads"]
    w = s.weights[s.layer]

    def take(i, r0, r1, score, v, before):
        z = s.lse[r0:r1].view(r1 - r0, H, -1).permute(1, 2, 0)[..., None]
        x = torch.exp(score - z).sum((1, 2))
        if before:
            w[s.prefix_sids[s.of[i]], :, :before] += x[:, :before]
        w[s.sids_list[i], :, :s.total[i]] += x[:, before:]

    _plain_rows(s, take)
    return w


def _plain_select(s):
    c = s.case
    L, H = c["layers"], c["kv_heads"]
    kept = torch.full((len(s.total), L, H, s.most), -1, dtype=torch.int32, device="cuda")
    for i, (sid, total, keep) in enumerate(zip(s.sids_list, s.total, s.keeps)):
        first = min(c["first"], keep)
        lo, hi = first, max(total - min(c["recent"], keep - first), first)      # those between them compete
        order = torch.sort(s.weights[:, sid, :, lo:hi], dim=-1, descending=True, stable=True).indices
        stay = torch.ones((L, H, total), dtype=torch.bool, device="cuda")
        stay[:, :, lo:hi] = False
        some = order[:, :, :keep - first - (total - hi)] + lo
        stay.scatter_(2, some, torch.ones_like(some, dtype=torch.bool))
        kept[i, :, :, :keep] = stay.nonzero()[:, 2].view(L, H, keep).to(torch.int32)
    return kept


def _plain_compact(s):
    c = s.case
    L, H, D, T = c["layers"], c["kv_heads"], c["head_dim"], c["page_tokens"]
    heads = torch.arange(H, device="cuda")[:, None]
    for i, (sid, total, keep) in enumerate(zip(s.sids_list, s.total, s.keeps)):
        if keep >= total:
            continue
        token = torch.arange(total, device="cuda")
        slots = s.table[sid].long()[token // T] * T + token % T
        for layer in range(L):
            at = s.kept[i, layer, :, :keep].long()
            for kv in range(2):
                x = s.kv[2 * layer + kv].view(-1, H, D)
                x[slots[:keep].expand(H, keep), heads] = x[slots[at], heads]
            w = s.weights[layer, sid]
            moved = w.gather(1, at)
            w[:, :total] = 0.0
            w[:, :keep] = moved
    return s.kv, s.weights


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    c = s.case
    kind = c["kind"]
    if not own:
        return {"shared": _plain_shared, "weights": _plain_weights, "select": _plain_select,
                "compact": _plain_compact}[kind](s)
    if kind == "shared":
        return s.batch.attention(s.layer, s.q, scale=s.scale, return_lse=c["lse"])
    if kind == "weights":
        s.batch.add_weights(s.layer, s.q, s.lse, s.weights[s.layer], last=c["last"], scale=s.scale)
        return s.weights[s.layer]
    if kind == "select":
        return s.pool.select_kept(s.sids, s.keeps_dev, s.weights, first=c["first"], last=c["recent"], most=s.most)
    s.pool.compact(s.sids, s.keeps_dev, s.kept, s.weights)
    return s.kv, s.weights


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    """In 64 bits, request by request and head by head, from the block tables as they were made."""
    c = case
    if c["kind"] == "select":
        return None
    global own
    mine, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = mine
    T, H, D, Hq, L = c["page_tokens"], c["kv_heads"], c["head_dim"], c["q_heads"], c["layers"]
    G = Hq // H
    if c["kind"] == "compact":
        if s.kv.numel() > 1 << 29:
            return None
        kv, w = s.kv.double(), s.weights.double()
        for sid, total, keep, kept in zip(s.sids_list, s.total, s.keeps, s.kept.cpu()):
            if keep == total:
                continue
            pages = s.table[sid].long()
            to = torch.arange(keep, device="cuda")
            for layer in range(L):
                for h in range(H):
                    j = kept[layer, h, :keep].long().cuda()
                    for x in (kv[2 * layer], kv[2 * layer + 1]):
                        rows = x[pages[j // T], j % T, h].clone()
                        x[pages[to // T], to % T, h] = rows
                    old = w[layer, sid, h, :total].clone()
                    w[layer, sid, h, :keep] = old[j]
                    w[layer, sid, h, keep:total] = 0
        return kv, w
    if 4 * D * sum(m * (t + (s.prefix[p] if p >= 0 else 0)) for m, t, p in zip(s.new, s.total, s.of)) * Hq > 4e12:
        return None
    out = torch.zeros((s.rows, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((s.rows, Hq), dtype=torch.float64, device="cuda")
    w = s.weights[s.layer].double() if c["kind"] == "weights" else None
    at = 0
    for i, (m, total) in enumerate(zip(s.new, s.total)):
        where = []                                # (page, place in it) of every key, in order
        for sid, count in ([(s.prefix_sids[s.of[i]], s.prefix[s.of[i]])] if s.of[i] >= 0 else []) + \
                [(s.sids_list[i], total)]:
            token = torch.arange(count, device="cuda")
            where.append((s.table[sid].long()[token // T], token % T))
        page, off = (torch.cat(x) for x in zip(*where))
        keys = len(page)
        begin = max(0, m - c["last"]) if c["last"] else 0
        step = max(1, (1 << 27) // max(keys, 1))
        for h in range(H):
            k, v = s.kv[2 * s.layer][page, off, h].double(), s.kv[2 * s.layer + 1][page, off, h].double()
            for g in range(h * G, (h + 1) * G):
                for a in range(begin, m, step):
                    b = min(m, a + step)
                    x = (s.q[at + a:at + b, g].double() @ k.T) * s.scale
                    p = torch.arange(keys - m + a, keys - m + b, device="cuda")
                    x[torch.arange(keys, device="cuda")[None] > p[:, None]] = -math.inf
                    if w is not None:
                        x = torch.exp(x - s.lse[at + a:at + b, g].double()[:, None]).sum(0)
                        if s.of[i] >= 0:
                            w[s.prefix_sids[s.of[i]], h, :keys - total] += x[:keys - total]
                        w[s.sids_list[i], h, :total] += x[keys - total:]
                        continue
                    z = torch.logsumexp(x, 1)
                    out[at + a:at + b, g] = torch.exp(x - z[:, None]) @ v
                    lse[at + a:at + b, g] = z
        at += m
    if w is not None:
        return w
    return (out, lse) if c["lse"] else out
