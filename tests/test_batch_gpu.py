"""Serving steps on resident KV: the plan's arrays, the write of K and V rows, what the calls refuse,
what they report, and what must not change a result (streams, strides, garbage in the pages, repetition)."""
import ctypes

import numpy as np
import pytest

from tests._attention import Step

pytestmark = pytest.mark.gpu


def _plan_by_hand(s, firsts=None, bad=()):
    """The plan's five arrays from the definition, one token at a time; bad: requests left out."""
    T, at = s.page, 0
    width = s.pool.max_blocks
    starts, kv_lens, tables = [0], [], np.full((s.n, width), -1, np.int32)
    positions, slots = np.full(s.rows, -1, np.int32), np.full(s.rows, -1, np.int64)
    for i in range(s.n):
        m = s.new[i]
        first = s.cached[i] if firsts is None or firsts[i] < 0 else firsts[i]
        if i not in bad:
            kv_lens.append(first + m)
            row = s.table[s.sids[i]]
            nb = -(-(first + m) // T)
            tables[i, :nb] = np.where(row[:nb] >= 0, row[:nb], -1)
            for t in range(m):
                p = first + t
                positions[at + t] = p
                slots[at + t] = int(row[p // T]) * T + p % T
        else:
            kv_lens.append(0)
        at += m
        starts.append(min(at, s.rows))
    return np.array(starts), np.array(kv_lens), tables, positions, slots


def _check_plan(s, want):
    b = s.batch
    got = (b.row_starts[:s.n + 1], b.kv_lens[:s.n], b.tables[:s.n], b.positions[:s.rows], b.slots[:s.rows])
    for name, g, w in zip(("row_starts", "kv_lens", "tables", "positions", "slots"), got, want):
        assert np.array_equal(g.cpu().numpy(), w), name


SMALL = dict(heads=1, group=2, dim=8)


@pytest.mark.parametrize("page", [1, 7, 16, 100])
@pytest.mark.parametrize("cached,new,pad", [([5], [1], 0), ([0, 16, 31, 3], [1, 0, 33, 2], 5), ([0], [0], 0),
                                            ([300] * 70, [1] * 70, 3), ([9, 0, 0, 2], [0, 0, 5, 0], 1)])
def test_plan(cached, new, pad, page):
    import torch
    s = Step(cached, new, pad=pad, page=page, **SMALL)
    try:
        for where in ("numpy", "device", "pinned"):
            conv = {"numpy": lambda x: x, "device": lambda x: torch.from_numpy(x).cuda(),
                    "pinned": lambda x: torch.from_numpy(x).pin_memory()}[where]
            s.batch.plan(conv(s.sids), conv(np.asarray(new, np.int32)), num_tokens=s.rows, max_len=max(new))
            assert s.pool.sync(raise_on_error=False) == 0
            _check_plan(s, _plan_by_hand(s))
    finally:
        s.close()


def test_plan_of_no_request():
    s = Step([3], [2], pad=4, **SMALL)
    try:
        s.batch.plan(np.zeros(0, np.int32), np.zeros(0, np.int32), num_tokens=6)
        assert s.pool.sync(raise_on_error=False) == 0
        assert int(s.batch.row_starts[0]) == 0
        assert (s.batch.positions[:6] == -1).all() and (s.batch.slots[:6] == -1).all()
        out, lse = s.batch.attention(0, s.q, return_lse=True)
        assert (out == 0).all() and (lse == -float("inf")).all()
        s.batch.plan(np.zeros(0, np.int32), np.zeros(0, np.int32))
        assert s.batch.attention(0, s.q[:0]).shape[0] == 0
        s.batch.write(0, s.q[:0, :1], s.q[:0, :1])
        assert s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()


def test_plan_of_a_prompts_chunks():
    """A context that grew at once is worked through in chunks, the queries of each at firsts."""
    s = Step([40], [100], heads=2, group=4, dim=64, max_tokens=100)
    try:
        want, mag, _, _ = s.attention64(0, 0.125)
        for a, b in ((0, 37), (37, 38), (38, 100)):
            s.batch.plan(s.sids, np.array([b - a], np.int32), np.array([40 + a], np.int32))
            out = s.batch.attention(0, s.q[a:b], scale=0.125)
            assert s.pool.sync(raise_on_error=False) == 0
            assert s.batch.positions[:b - a].tolist() == list(range(40 + a, 40 + b))
            assert int(s.batch.kv_lens[0]) == 40 + b
            bound = 2.0 ** -8 * want[a:b].abs() + 2.0 ** -7 * mag[a:b] + 1e-5
            assert ((out.double() - want[a:b]).abs() <= bound).all()
    finally:
        s.close()


@pytest.mark.parametrize("what", ["sid", "negative", "longer", "rows", "first", "max_len"])
def test_requests_left_out(what):
    """A request that breaks a rule is reported and left out, and the others go on."""
    from paper_2606_22983_gb300 import lv
    s = Step([20, 50, 7], [3, 2, 4], heads=2, group=4, dim=64, pad=2)
    try:
        sids, lens, firsts, max_len = s.sids.copy(), np.array([3, 2, 4], np.int32), np.full(3, -1, np.int32), 4
        bad = 1
        if what == "sid":
            sids[1] = s.pool.S
        elif what == "negative":
            lens[1], s.new[1], s.rows = -5, 0, s.rows - 2
        elif what == "longer":
            lens[1], s.new[1], s.rows = 53, 53, s.rows + 51
        elif what == "rows":
            bad, s.rows = 2, 8                   # the last request's rows do not fit
        elif what == "first":
            firsts[1] = 51                       # 51 + 2 is past the context of 52
        elif what == "max_len":
            lens[2], max_len, bad = 4, 3, 2
        s.batch.max_tokens
        if s.rows > s.batch.max_tokens:
            s.close()
            s = Step([20, 50, 7], [3, 2, 4], heads=2, group=4, dim=64, pad=2, max_tokens=80)
            s.new[1], s.rows = 53, 3 + 53 + 4 + 2
        s.batch.plan(sids, lens, firsts, num_tokens=s.rows, max_len=60 if what == "longer" else max_len)
        st = s.pool.stats()
        assert st["error"] == lv.LV_ERR_BOUNDS and st["error_detail"] == bad
        s.pool.clear_error()
        want = _plan_by_hand(s, bad=(bad,))
        if what == "rows":
            want[3][5:], want[4][5:] = -1, -1
        _check_plan(s, want)
        import torch
        q = torch.randn((s.rows, 8, 64), device="cuda").to(torch.bfloat16)
        out, lse = s.batch.attention(1, q, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        live = torch.from_numpy(want[3] >= 0)
        assert (out[~live.cuda()] == 0).all() and torch.isinf(lse[~live.cuda()]).all()
        assert torch.isfinite(out).all() and (out[live.cuda()] != 0).any() and torch.isfinite(lse[live.cuda()]).all()
    finally:
        s.close()


def test_blocks_in_the_host_tier():
    """A visible block that is not in HBM is reported and its request left out; under a window the
    blocks that no row sees may be in the host tier."""
    from paper_2606_22983_gb300 import lv
    away = {(0, 3)}
    s = Step([200, 40], [1, 1], heads=2, group=4, dim=64, absent=away)
    try:
        s.plan()
        st = s.pool.stats()
        assert st["error"] == lv.LV_ERR_STATE and st["error_detail"] == 0
        s.pool.clear_error()
        _check_plan(s, _plan_by_hand(s, bad=(0,)))
        out = s.batch.attention(0, s.q)
        assert s.pool.sync(raise_on_error=False) == 0
        assert (out[0] == 0).all() and (out[1] != 0).any()
    finally:
        s.close()
    # keys 0..16 and the last 100 of 331 are seen: blocks 2 to 13 may be away, not block 14
    for new in ([1], [30]):
        s = Step([331 - new[0]], new, heads=2, group=4, dim=128, window=100, sinks=17,
                 absent={(0, b) for b in range(2, (331 - new[0] - 99) // 16)})
        try:
            s.plan()
            assert s.pool.sync(raise_on_error=False) == 0
            out, lse = s.batch.attention(1, s.q, return_lse=True)
            s.check(out, lse, 1, 128 ** -0.5)
        finally:
            s.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("source", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", ["dense", "fused", "odd", "reversed"])
def test_write(dtype, source, layout):
    import torch
    kinds = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    cached, new, H, D = [0, 15, 16, 33], [1, 20, 0, 7], 3, 24
    s = Step(cached, new, heads=H, group=1, dim=D, pad=2, dtype=kinds[dtype])
    try:
        s.plan()
        x = torch.randn((2, s.rows, H, D), device="cuda") * 100
        if layout == "dense":
            k, v = x.to(kinds[source])
        elif layout == "fused":          # a projection's row: queries, K and V heads side by side
            row = torch.zeros((s.rows, 4 * H, D), device="cuda", dtype=kinds[source])
            row[:, H:2 * H], row[:, 3 * H:] = x[0], x[1]
            k, v = row[:, H:2 * H], row[:, 3 * H:]
        elif layout == "odd":            # rows of an odd length from an odd element on
            flat = torch.zeros((2, s.rows * (H * D + 5) + 1), device="cuda", dtype=kinds[source])
            k, v = (f[1:].as_strided((s.rows, H, D), (H * D + 5, D, 1), 1 + f.storage_offset()) for f in flat)
            k.copy_(x[0]), v.copy_(x[1])
        else:                            # heads outermost
            k, v = (y.to(kinds[source]).transpose(0, 1).contiguous().transpose(0, 1) for y in x)
        before = s.kv.clone()
        s.batch.write(1, k, v)
        assert s.pool.sync(raise_on_error=False) == 0
        _, _, _, positions, slots = _plan_by_hand(s)
        want = before
        for i, slot in enumerate(slots):
            if slot >= 0:
                for kv, y in enumerate((k, v)):
                    want[2 + kv].view(-1, H, D)[slot] = y[i].float().to(kinds[dtype])
        assert torch.equal(s.kv.view(torch.int16), want.view(torch.int16))
    finally:
        s.close()


def test_written_rows_are_attended():
    """Both calls of a step, layer by layer, in a captured graph that is replayed with new values."""
    import torch
    s = Step([100, 0, 37], [3, 18, 1], heads=2, group=4, dim=128, layers=3)
    try:
        s.plan()
        k, v = (torch.randn((s.rows, 2, 128), device="cuda") for _ in range(2))
        outs = [torch.empty_like(s.q) for _ in range(3)]

        def step():
            for layer in range(3):
                s.batch.write(layer, k, v)
                s.batch.attention(layer, s.q, out=outs[layer])

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step()
        torch.cuda.synchronize()
        for _ in range(2):
            k.normal_(), v.normal_(), s.q.normal_()
            g.replay()
            torch.cuda.synchronize()
            assert s.pool.sync(raise_on_error=False) == 0
            for layer in range(3):
                s.check(outs[layer], None, layer, 128 ** -0.5)
    finally:
        s.close()


def test_rows_with_a_clean_host_copy_are_not_written():
    from paper_2606_22983_gb300 import lv
    import torch
    s = Step([20], [2], heads=1, group=1, dim=8, tiers=lv.LV_TIERS_INCLUSIVE, host_pages=8, max_tokens=64)
    try:
        # evicted and loaded back: block 1, where the new tokens lie, keeps a clean copy
        sid = int(s.sids[0])
        victims, n = s.pool.select(0, 2)
        assert n == 2
        s.pool.exchange(victims, 2, sid, None, 0)
        blks, n = s.pool.blocks(sid, 1)
        s.pool.exchange(None, 0, sid, blks, n)
        s.pool.sync()
        s.plan()
        assert s.pool.sync(raise_on_error=False) == 0
        slots = s.batch.slots[:2].cpu().numpy()
        assert (slots <= -2).all()
        kv = s.kv.clone()
        k = torch.ones((2, 1, 8), device="cuda")
        s.batch.write(0, k, k)
        st = s.pool.stats()
        assert st["error"] == lv.LV_ERR_STATE and st["error_detail"] in (0, 1)
        s.pool.clear_error()
        assert torch.equal(s.kv.view(torch.int16), kv.view(torch.int16))
        table = s.pool.tables()[0][sid]
        assert (-(slots + 2) // 16 == table[1]).all()
        # a context that grows drops the copy (lv_session_append), and its rows may be written
        s.pool.append(sid, 3)
        s.batch.plan(s.sids, np.array([3], np.int32))
        assert s.pool.sync(raise_on_error=False) == 0
        k = torch.ones((3, 1, 8), device="cuda")
        s.batch.write(0, k, k)
        assert s.pool.sync(raise_on_error=False) == 0
        at = s.batch.slots[:3]
        assert (at >= 0).all() and (s.kv[0].view(-1, 8)[at] == 1).all() and (s.kv[1].view(-1, 8)[at] == 1).all()
    finally:
        s.close()


@pytest.mark.parametrize("new", [[1, 1], [90, 3]])
def test_strides_and_streams(new):
    """Queries and outputs in other orders, odd strides and alignments, on another stream."""
    import torch
    s = Step([70, 400], new, heads=2, group=4, dim=96, pad=1)
    try:
        s.plan()
        base, lse0 = s.batch.attention(1, s.q, return_lse=True)
        s.check(base, lse0, 1, 96 ** -0.5)
        n, Hq, D = s.q.shape
        odd = torch.zeros(n * (Hq * D + 7) + 1, device="cuda", dtype=s.q.dtype)[1:].as_strided(
            (n, Hq, D), (Hq * D + 7, D, 1), 1)
        odd.copy_(s.q)
        heads_first = s.q.transpose(0, 1).contiguous().transpose(0, 1)
        same = s.q[:, :1].expand(n, Hq, D)                     # one query for every head: stride 0
        side = torch.cuda.Stream()
        for q in (odd, heads_first):
            for shape in ("dense", "odd", "heads_first"):
                if shape == "dense":
                    out = torch.empty_like(base)
                elif shape == "odd":
                    out = torch.zeros(n * (Hq * D + 9) + 1, device="cuda", dtype=s.q.dtype)[1:].as_strided(
                        (n, Hq, D), (Hq * D + 9, D, 1), 1)
                else:
                    out = torch.empty((Hq, n, D), device="cuda", dtype=s.q.dtype).transpose(0, 1)
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    s.batch.attention(1, q, out=out)
                torch.cuda.current_stream().wait_stream(side)
                assert torch.equal(out, base), shape
                s.batch.attention(1, q, out=out, stream=side)
                side.synchronize()
                assert torch.equal(out, base), shape
        out = s.batch.attention(1, same)
        assert s.pool.sync(raise_on_error=False) == 0
        s.check(out, None, 1, 96 ** -0.5, q=same)
    finally:
        s.close()


@pytest.mark.parametrize("cached,new", [([30000], [1]), ([900] * 20, [1] * 20), ([12000, 50], [200, 1])])
def test_same_bits_every_time(cached, new):
    """Pieces are joined in their own order, whichever ends last."""
    import torch
    s = Step(cached, new, heads=2, group=8, dim=128, sharp=2.0)
    try:
        s.plan()
        first = s.batch.attention(0, s.q, return_lse=True)
        for _ in range(20):
            again = s.batch.attention(0, s.q, return_lse=True)
            assert all(torch.equal(a, b) for a, b in zip(first, again))
    finally:
        s.close()


def test_infinite_and_extreme_scores():
    """Scores past the 16-bit range, and rows whose scores are all very low."""
    import torch
    for new in ([1], [100]):
        for dtype in (torch.bfloat16, torch.float16):
            s = Step([300], new, heads=1, group=4, dim=64, dtype=dtype)
            try:
                s.plan()
                big = 60.0 if dtype == torch.float16 else 1e4
                q = s.q * big
                out, lse = s.batch.attention(0, q, scale=1.0, return_lse=True)
                s.check(out, lse, 0, 1.0, q=q)
                q = -s.kv[0][s.table[s.sids[0], 0], 0, :1].expand(new[0], 4, 64) * big      # key 0 scores lowest
                out, lse = s.batch.attention(0, q, scale=1.0, return_lse=True)
                s.check(out, lse, 0, 1.0, q=q)
            finally:
                s.close()


def test_far_pages():
    """K and V arrays of more than 2^32 bytes each, the context in their last pages."""
    import torch
    from paper_2606_22983_gb300.batch import KVBatch
    from paper_2606_22983_gb300.pool import KVPool
    pages, T, H, D = (1 << 32) // 16384 + 100, 16, 4, 128
    kv = torch.zeros((2, pages, T, H, D), dtype=torch.bfloat16, device="cuda")
    pool = KVPool(layers=1, kv_heads=H, head_dim=D, max_sessions=2, max_blocks=80, hbm_pages=pages,
                  hbm_budget_pages=pages, host_pages=0, kv=kv.view(torch.uint8).view(2, pages, T * H * D * 2))
    try:
        table = np.full((2, 80), -1, np.int32)
        table[1] = np.arange(pages - 80, pages)[::-1]
        for n in (1, 200):
            ctx = 1000 + n
            row = table.copy()
            row[1, -(-ctx // T):] = -1
            pool.import_placement(row, np.array([0, ctx], np.int32))
            b = KVBatch(pool, q_heads=32, max_requests=1, max_tokens=n)
            kv[:, pages - 80:] = 0
            b.plan([1], [n])
            k, v = (torch.randn((n, H, D), device="cuda").bfloat16() for _ in range(2))
            b.write(0, k, v)
            assert pool.sync(raise_on_error=False) == 0
            slots = b.slots[:n].cpu().numpy()
            pos = np.arange(1000, ctx)
            assert np.array_equal(slots, table[1][pos // T].astype(np.int64) * T + pos % T)
            page = torch.from_numpy(slots // T).cuda()
            assert torch.equal(kv[0][page, torch.from_numpy(slots % T).cuda()], k)
            # every cached key is zero: each row averages V over its context
            q = torch.zeros((n, 32, D), device="cuda", dtype=torch.bfloat16)
            out = b.attention(0, q).double()
            want = v.double().cumsum(0) / torch.arange(1001, ctx + 1, device="cuda")[:, None, None]
            want = want.repeat_interleave(8, 1)
            assert pool.sync(raise_on_error=False) == 0
            assert ((out - want).abs() <= 2.0 ** -7 * want.abs() + 1e-6).all()
    finally:
        pool.close()


def _desc(lv, s, **kw):
    b = s.batch
    d = dict(num_q_heads=8, max_requests=4, max_tokens=16, dtype=lv.LV_BF16, window=0, sinks=0,
             row_starts=b.row_starts.data_ptr(), kv_lens=b.kv_lens.data_ptr(), tables=b.tables.data_ptr(),
             positions=b.positions.data_ptr(), slots=b.slots.data_ptr())
    d.update(kw)
    return lv.lv_batch_desc(**d)


def test_refusals():
    import torch
    from paper_2606_22983_gb300 import lv
    from paper_2606_22983_gb300.batch import KVBatch
    from paper_2606_22983_gb300.pool import KVPool
    s = Step([20, 30], [1, 2], heads=2, group=4, dim=64, max_requests=4, max_tokens=16)
    host = np.zeros(64, np.int64)
    try:
        for kw in (dict(num_q_heads=0), dict(num_q_heads=1), dict(num_q_heads=7), dict(num_q_heads=2 * 257),
                   dict(max_requests=0), dict(max_requests=4097), dict(max_tokens=0), dict(max_tokens=(1 << 24) + 1),
                   dict(max_tokens=1 << 24, num_q_heads=256), dict(dtype=0), dict(dtype=lv.LV_F32), dict(window=-1),
                   dict(window=(1 << 30) + 1), dict(sinks=-1), dict(sinks=(1 << 30) + 1),
                   dict(reserved=(ctypes.c_int32 * 2)(0, 1)), dict(row_starts=None), dict(tables=0),
                   dict(kv_lens=s.batch.kv_lens.data_ptr() + 2), dict(slots=s.batch.slots.data_ptr() + 4),
                   dict(positions=host.ctypes.data)):
            with pytest.raises(lv.LvError) as e:
                lv.lv_batch_create(s.pool.handle, _desc(lv, s, **kw))
            assert e.value.status == lv.LV_ERR_INVALID, kw
        for shape in (dict(elem_bytes=1, head_dim=16), dict(elem_bytes=4, head_dim=16), dict(elem_bytes=2, head_dim=4),
                      dict(elem_bytes=2, head_dim=264)):
            p = KVPool(layers=1, kv_heads=2, max_sessions=1, max_blocks=1, hbm_pages=1, hbm_budget_pages=1,
                       host_pages=0, **shape)
            with pytest.raises(lv.LvError):
                KVBatch(p, q_heads=2, max_requests=1, max_tokens=1)
            p.close()
        with pytest.raises(ValueError):
            KVBatch(s.pool, q_heads=2, max_requests=1, max_tokens=1, dtype=torch.float32)

        b, L, null = s.batch, lv.lib(), None
        k = torch.zeros((3, 2, 64), device="cuda", dtype=torch.bfloat16)
        q = torch.zeros((3, 8, 64), device="cuda", dtype=torch.bfloat16)
        with pytest.raises(lv.LvError):                      # nothing planned yet
            b.attention(0, q)
        with pytest.raises(lv.LvError):
            b.write(0, k, k)
        plan = lambda *a: L.lv_batch_plan(b.handle, *a, None)
        sids, lens = torch.from_numpy(s.sids).cuda(), torch.tensor([1, 2], dtype=torch.int32, device="cuda")
        p_sids, p_lens = sids.data_ptr(), lens.data_ptr()
        for a in ((p_sids, null, p_lens, -1, 3, 2), (p_sids, null, p_lens, 5, 3, 2), (null, null, p_lens, 2, 3, 2),
                  (p_sids, null, null, 2, 3, 2), (p_sids, null, p_lens, 2, -1, 2), (p_sids, null, p_lens, 2, 17, 2),
                  (p_sids, null, p_lens, 2, 3, -1)):
            assert plan(*a) == lv.LV_ERR_INVALID, a
        with pytest.raises(ValueError):
            b.plan(sids, lens)                               # lengths on the device and no num_tokens
        with pytest.raises(ValueError):
            b.plan(sids, lens[:1], num_tokens=3)
        with pytest.raises(ValueError):
            b.plan(sids.long(), lens, num_tokens=3)
        s.plan()

        def heads(x, **kw):
            h = lv.lv_heads(data=x.data_ptr(), row_stride=x.stride(0), head_stride=x.stride(1), dtype=lv.LV_BF16)
            for n, y in kw.items():
                setattr(h, n, y)
            return ctypes.byref(h)

        bad = (dict(data=None), dict(data=k.data_ptr() + 1), dict(data=host.ctypes.data), dict(dtype=0), dict(dtype=4),
               dict(reserved=1), dict(row_stride=1 << 40), dict(head_stride=-(1 << 40)))
        for kw in bad:
            assert L.lv_kv_write(b.handle, 0, heads(k, **kw), heads(k), None) == lv.LV_ERR_INVALID, kw
            assert L.lv_kv_write(b.handle, 0, heads(k), heads(k, **kw), None) == lv.LV_ERR_INVALID, kw
            assert L.lv_attention(b.handle, 0, heads(q, **kw), heads(q), None, 1.0, None) == lv.LV_ERR_INVALID, kw
            assert L.lv_attention(b.handle, 0, heads(q), heads(q, **kw), None, 1.0, None) == lv.LV_ERR_INVALID, kw
        assert L.lv_kv_write(b.handle, 0, None, heads(k), None) == lv.LV_ERR_INVALID
        for layer in (-1, 2):
            assert L.lv_kv_write(b.handle, layer, heads(k), heads(k), None) == lv.LV_ERR_INVALID
            assert L.lv_attention(b.handle, layer, heads(q), heads(q), None, 1.0, None) == lv.LV_ERR_INVALID
        for scale in (0.0, -1.0, float("inf"), float("nan")):
            assert L.lv_attention(b.handle, 0, heads(q), heads(q), None, scale, None) == lv.LV_ERR_INVALID
        for dtype in (lv.LV_F16, lv.LV_F32):
            assert L.lv_attention(b.handle, 0, heads(q, dtype=dtype), heads(q), None, 1.0, None) == lv.LV_ERR_INVALID
        assert L.lv_attention(b.handle, 0, heads(q), heads(q), host.ctypes.data, 1.0, None) == lv.LV_ERR_INVALID
        for x in (q[:2], q[:, :7], q[:, :, :32], q.transpose(1, 2), q.float().double(), q.cpu(), q[0]):
            with pytest.raises(ValueError):
                b.attention(0, x)
        assert s.pool.sync(raise_on_error=False) == 0        # and none of it left a mark
        s.check(b.attention(0, s.q), None, 0, 0.125)
    finally:
        s.close()


@pytest.mark.parametrize("n", [255, 256, 257, 700])
def test_plan_of_many_requests(n):
    """On both sides of the size from which the plan is two kernels."""
    rng = np.random.default_rng(n)
    new = rng.integers(0, 4, n)
    new[rng.integers(0, n)] = 37
    s = Step(rng.integers(0, 90, n).tolist(), new.tolist(), heads=2, group=2, dim=16, pad=3)
    try:
        s.plan()
        assert s.pool.sync(raise_on_error=False) == 0
        _check_plan(s, _plan_by_hand(s))
        out, lse = s.batch.attention(1, s.q, return_lse=True)
        s.check(out, lse, 1, 0.25)
    finally:
        s.close()
