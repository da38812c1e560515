"""Choosing the tokens that sessions keep, moving their K and V, and cutting the contexts: each against its
definition, with what the calls refuse and report."""
import ctypes

import numpy as np
import pytest

from tests._kept import Kept

pytestmark = pytest.mark.gpu


def _i32(x):
    return np.asarray(x, np.int32)


def _chosen(s, keeps, got, first, last, requests=None):
    for k, i in enumerate(range(len(s.total)) if requests is None else requests):
        want = s.choose(i, keeps[k], first, last)
        n = want.shape[2]
        assert np.array_equal(got[k, :, :, :n], want), i
        assert (got[k, :, :, n:] == -1).all()


CHOICES = [
    # (contexts, kept, first, last)
    ([1], [1], 0, 0), ([1], [0], 3, 3), ([0, 5], [4, 2], 1, 1), ([100], [100], 4, 10), ([100], [130], 4, 10),
    ([100, 37, 513, 16], [50, 36, 100, 1], 4, 32), ([700], [40], 30, 30), ([700], [40], 50, 30), ([700], [41], 0, 40),
    ([2048, 2049, 511, 512, 513], [1024, 7, 510, 511, 1], 0, 0), ([30000], [1234], 33, 700), ([70001], [20000], 4, 128),
]


@pytest.mark.parametrize("total,keeps,first,last", CHOICES)
def test_choice(total, keeps, first, last):
    s = Kept(total, heads=1, dim=8)
    try:
        got = s.pool.select_kept(s.sids, _i32(keeps), s.weights, first=first, last=last)
        assert s.pool.sync(raise_on_error=False) == 0
        _chosen(s, keeps, got.cpu().numpy(), first, last)
    finally:
        s.close()


@pytest.mark.parametrize("what", ["equal", "zeros", "infinities", "nan", "negative", "close"])
def test_choice_of_odd_weights(what):
    import torch
    s = Kept([3000, 600], heads=2, dim=8)
    try:
        w, g = s.weights, torch.Generator(device="cuda").manual_seed(1)
        pick = torch.rand(w.shape, generator=g, device="cuda")
        if what == "equal":
            w.fill_(0.25)
        elif what == "zeros":
            w[pick < 0.9] = 0.0
            w[pick < 0.4] = -0.0
        elif what == "infinities":
            w[pick < 0.5] = float("inf")
            w[pick < 0.2] = -float("inf")
        elif what == "nan":
            w[pick < 0.3] = float("nan")
            w[pick < 0.2] = float("inf")
            w[pick < 0.1] = torch.tensor(-4194303, dtype=torch.int32).view(torch.float32).item()     # a NaN with its sign set
        elif what == "negative":
            w.sub_(0.05)
        else:      # keys that differ in their lowest bits only, subnormal ones among them
            w.copy_(((pick * 40).to(torch.int32) + torch.where(pick < 0.5, 1, 0x3f800000).to(torch.int32)).view(torch.float32))
        for keeps in ([1000, 599], [17, 300]):
            got = s.pool.select_kept(s.sids, _i32(keeps), w, first=2, last=9)
            assert s.pool.sync(raise_on_error=False) == 0
            _chosen(s, keeps, got.cpu().numpy(), 2, 9)
    finally:
        s.close()


def test_choice_by_strided_weights_of_some_sessions():
    import torch
    s = Kept([200, 90, 40], heads=3, dim=8, layers=4)
    try:
        wide = torch.full((4, 2, s.pool.S, 5, s.tokens + 7), 9.0, device="cuda").transpose(0, 1)[1][:, :, 1:4, 3:]
        wide[..., :s.tokens] = s.weights
        for conv in (lambda x: x, lambda x: torch.from_numpy(x).cuda(), lambda x: torch.from_numpy(x).pin_memory()):
            got = s.pool.select_kept(conv(s.sids[[2, 0, 2]]), conv(_i32([10, 30, 39])), wide, first=1, last=2, most=45)
            assert s.pool.sync(raise_on_error=False) == 0 and got.shape == (3, 4, 3, 45)
            _chosen(s, [10, 30, 39], got.cpu().numpy(), 1, 2, [2, 0, 2])
    finally:
        s.close()


def test_choices_left_out():
    from paper_2606_22983_gb300 import lv
    s = Kept([200, 90, 40], heads=1, dim=8)
    try:
        for sids, keeps, most, short in (([s.pool.S, 1], [3, 3], 5, False), ([-1, 1], [3, 3], 5, False),
                                         ([0, 1], [-1, 3], 5, False), ([0, 1], [6, 3], 5, False), ([0, 1], [3, 3], 5, True)):
            x = s.sids[:2].copy()
            if sids[0] not in (0,):
                x[0] = sids[0]
            w = s.weights[..., :199] if short else s.weights
            got = s.pool.select_kept(x, _i32(keeps), w, most=most).cpu().numpy()
            assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_BOUNDS and s.pool.stats()["error_detail"] == 0
            s.pool.clear_error()
            assert (got[0] == -1).all()
            _chosen(s, [3], got[1:], 0, 0, [1])
    finally:
        s.close()


MOVES = [
    # (contexts, kept, K and V's shape)
    ([100], [33], dict()), ([1, 2, 17, 700], [1, 1, 16, 350], dict()), ([513], [512], dict(dim=128, heads=4)),
    ([900, 30, 0, 64], [1, 0, 0, 64], dict(dim=96, heads=3)), ([300, 200], [150, 20], dict(dim=8, heads=1, page=7)),
    ([300], [99], dict(dim=12, heads=4, page=1, elem=1)), ([300], [100], dict(dim=5, heads=2, elem=4, page=8)),
    ([5000] * 3, [2500, 4999, 40], dict(dim=64, heads=1, layers=1)), ([2000], [700], dict(dim=128, heads=8, layers=6, page=64)),
    ([64] * 200, [1 + i % 64 for i in range(200)], dict(dim=16, heads=1)), ([40], [20], dict(dim=2048, heads=1, layers=1)),
]


@pytest.mark.parametrize("total,keeps,shape", MOVES)
def test_moves(total, keeps, shape):
    import torch
    s = Kept(total, slack=5, **shape)
    try:
        kept = [s.choose(i, keeps[i], 1, 3) for i in range(len(total))]
        most = max(max(keeps), 1)
        lists = np.full((len(total), s.layers, s.heads, most), -1, np.int32)
        for i, x in enumerate(kept):
            lists[i, :, :, :x.shape[2]] = x
        kv, w = s.moved(range(len(total)), keeps, kept)
        lens = s.pool.compact(s.sids, _i32(keeps), torch.from_numpy(lists).cuda(), s.weights)
        assert s.pool.sync(raise_on_error=False) == 0
        assert lens.tolist() == [min(k, t) for k, t in zip(keeps, total)]
        assert np.array_equal(s.kv.cpu().numpy(), kv)
        assert np.array_equal(s.weights.cpu().numpy().view(np.int32), w.view(np.int32))
        # the tables are as they were; then the contexts end
        assert np.array_equal(s.pool.tables()[0], s.table)
        s.pool.truncate(s.sids, lens)
        assert s.pool.sync(raise_on_error=False) == 0
        _check_cut(s, lens.tolist())
    finally:
        s.close()


def _check_cut(s, lens):
    """Tables, owners, counts and allocations of contexts cut to lens."""
    tables, hbm, host = s.pool.tables()
    want = s.table.copy()
    for sid, n in zip(s.sids, lens):
        want[sid, -(-n // s.page):] = -1
    assert np.array_equal(tables, want)
    owned = np.full(len(hbm), -1, np.int64)
    for sid, b in zip(*np.nonzero(want >= 0)):
        owned[want[sid, b]] = (sid << 16) | b
    assert np.array_equal(hbm.astype(np.int64), owned)
    a, b = s.pool.counts()
    assert np.array_equal(a, (want >= 0).sum(1)) and np.array_equal(b, (want <= -2).sum(1))
    st = s.pool.stats()
    assert st["hbm_allocated"] == (want >= 0).sum()
    assert st["host_allocated"] - st["clean_copies"] == (want <= -2).sum()
    ctx = s.pool.get_sessions()["ctx_tokens"]
    for i, sid in enumerate(s.sids):
        assert ctx[sid] == lens[i]


def test_moves_without_weights_and_by_pageable_lists():
    s = Kept([300], dim=64)
    try:
        kept = s.choose(0, 100, 4, 4)
        kv, _ = s.moved([0], [100], [kept], weights=False)
        w = s.weights.clone()
        lens = s.pool.compact(s.sids, _i32([100]), kept[None])
        assert s.pool.sync(raise_on_error=False) == 0 and lens.tolist() == [100]
        assert np.array_equal(s.kv.cpu().numpy(), kv) and (w == s.weights).all()
    finally:
        s.close()


@pytest.mark.parametrize("what", ["order", "twice", "past", "negative", "sid", "length", "most", "absent", "again", "tokens"])
def test_moves_left_out(what):
    """A request that breaks a rule in one list of one head moves nothing, in no layer; the others move."""
    from paper_2606_22983_gb300 import lv
    host = {(1, 3)} if what == "absent" else ()
    s = Kept([200, 90, 40], heads=2, dim=64, host=host, room=4)
    try:
        keeps = [50, 30, 20]
        kept = [s.choose(i, keeps[i], 1, 2) for i in range(3)]
        lists = np.full((3, 2, 2, 60), -1, np.int32)
        for i, x in enumerate(kept):
            lists[i, :, :, :x.shape[2]] = x
        sids, code, weights = s.sids.copy(), lv.LV_ERR_BOUNDS, s.weights
        if what == "order":
            lists[1, 1, 0, [3, 4]] = lists[1, 1, 0, [4, 3]]
        elif what == "twice":
            lists[1, 0, 1, 7] = lists[1, 0, 1, 6]
        elif what == "past":
            lists[1, 1, 1, 29] = 90
        elif what == "negative":
            lists[1, 0, 0, 0] = -1
        elif what == "sid":
            sids[1] = s.pool.S
        elif what == "length":
            keeps[1] = -1
        elif what == "most":
            keeps[1] = 61
        elif what == "absent":
            code = lv.LV_ERR_STATE
        elif what == "again":
            sids[1], code = sids[0], lv.LV_ERR_DOUBLE_MAP
        done = [0, 2]
        if what == "tokens":
            weights, done = s.weights[..., :120], [1, 2]      # too few for the first session alone
        kv, w = s.moved(done, [keeps[i] for i in done], kept)
        import torch
        lens = s.pool.compact(sids, _i32(keeps), torch.from_numpy(lists).cuda(), weights)
        assert s.pool.sync(raise_on_error=False) == code
        assert s.pool.stats()["error_detail"] == (0 if what == "tokens" else 1)
        assert lens.tolist() == ([-1, 30, 20] if what == "tokens" else [50, -1, 20])
        assert np.array_equal(s.kv.cpu().numpy(), kv) and np.array_equal(s.weights.cpu().numpy(), w)
        s.pool.clear_error()
        s.pool.truncate(s.sids, lens)
        assert s.pool.sync(raise_on_error=False) == 0
        left = [n if n >= 0 else t for n, t in zip(lens.tolist(), s.total)]
        ctx = s.pool.get_sessions()["ctx_tokens"]
        assert [int(ctx[x]) for x in s.sids] == left
    finally:
        s.close()


def test_cut():
    """Contexts of either tier end where they are told to; what is no longer, or below zero, stays."""
    s = Kept([100, 33, 64, 7, 50], dim=8, heads=1, host={(0, 2), (0, 6), (2, 0), (4, 1), (4, 2), (4, 3)}, room=9)
    try:
        s.pool.truncate(s.sids, _i32([40, 33, 0, -1, 17]))
        assert s.pool.sync(raise_on_error=False) == 0
        _check_cut(s, [40, 33, 0, 7, 17])
        # the freed pages are given out again, the lowest first
        free = sorted(set(range(s.pool.hbm_pages)) - set(s.pool.tables()[0][s.pool.tables()[0] >= 0].tolist()))
        pages = s.pool.append(int(s.sids[2]), 20)
        assert s.pool.sync(raise_on_error=False) == 0 and pages.tolist() == free[:2]
    finally:
        s.close()


def test_cuts_left_out():
    from paper_2606_22983_gb300 import lv
    s = Kept([100, 33], dim=8, heads=1)
    try:
        s.pool.truncate(_i32([s.sids[0], s.pool.S, s.sids[1]]), _i32([20, 3, 5]))
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_BOUNDS and s.pool.stats()["error_detail"] == 1
        s.pool.clear_error()
        _check_cut(s, [20, 5])
        s.pool.truncate(_i32([s.sids[0], s.sids[0]]), _i32([10, 3]))
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_DOUBLE_MAP and s.pool.stats()["error_detail"] == 1
        s.pool.clear_error()
        _check_cut(s, [10, 5])
        s.pool.truncate(_i32([s.sids[0], s.sids[0], -5]), _i32([-1, 3, -1]))
        assert s.pool.sync(raise_on_error=False) == 0
        _check_cut(s, [3, 5])
    finally:
        s.close()


def test_clean_copies():
    """Blocks that are moved to, and freed ones, have no clean host copy any more."""
    from paper_2606_22983_gb300 import lv
    s = Kept([96, 64], dim=64, heads=1, host={(0, 0), (0, 1), (0, 5), (1, 2)}, room=12, tiers=lv.LV_TIERS_INCLUSIVE)
    try:
        for i in (0, 1):
            lv.lv_make_resident(s.pool.handle, int(s.sids[i]), 1000, 0, 0, -1, None, None, None, None, None, None, None)
        assert s.pool.sync(raise_on_error=False) == 0 and s.pool.stats()["clean_copies"] == 4
        kept = s.choose(0, 20, 0, 5)
        s.table = s.pool.tables()[0].copy()
        lens = s.pool.compact(s.sids[:1], _i32([20]), kept[None], s.weights)
        st = s.pool.stats()
        assert st["clean_copies"] == 2 and st["clean_dropped"] == 2 and lens.tolist() == [20]
        s.pool.truncate(s.sids[:1], lens)
        st = s.pool.stats()
        assert st["clean_copies"] == 1 and st["host_allocated"] == 1 and s.pool.sync(raise_on_error=False) == 0
        _check_cut(s, [20, 64])
    finally:
        s.close()


def test_refusals():
    import torch
    from paper_2606_22983_gb300 import lv
    s = Kept([50], dim=8, heads=1)
    try:
        h, w, sids, one = s.pool.handle, s.pool._put_weights(lv.lv_weights(), s.weights), s.sids, _i32([10])
        out = torch.zeros((1, 2, 1, 10), dtype=torch.int32, device="cuda")
        sel = lambda **k: (lambda d: lv.lv_select_kept(h, d["w"], d["sids"], d["keeps"], d["n"], d["first"], d["last"], d["kept"],
                                                       d["most"], None))({**dict(w=w, sids=sids, keeps=one, n=1, first=0, last=0,
                                                                                 kept=out, most=10), **k})
        null = lv.lv_weights(data=0, tokens=3)
        host = lv.lv_weights(data=np.zeros(4, np.float32).ctypes.data, tokens=1)
        odd = lv.lv_weights(data=s.weights.data_ptr() + 2, tokens=1)
        far = lv.lv_weights(data=s.weights.data_ptr(), layer_stride=1 << 39, tokens=1)
        res = lv.lv_weights(data=s.weights.data_ptr(), tokens=1, reserved=1)
        neg = lv.lv_weights(data=s.weights.data_ptr(), tokens=-1)
        for k in (dict(n=-1), dict(n=4097), dict(first=-1), dict(last=-1), dict(most=0), dict(kept=None), dict(sids=None),
                  dict(keeps=None), dict(w=null), dict(w=host), dict(w=odd), dict(w=far), dict(w=res), dict(w=neg)):
            with pytest.raises(lv.LvError) as e:
                sel(**k)
            assert e.value.status == lv.LV_ERR_INVALID, k
        lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        for a in ((sids, one, -1, out, 10, w, lens), (sids, one, 4097, out, 10, w, lens), (sids, one, 1, out, 0, w, lens),
                  (None, one, 1, out, 10, w, lens), (sids, None, 1, out, 10, w, lens), (sids, one, 1, None, 10, w, lens),
                  (sids, one, 1, out, 10, odd, lens), (sids, one, 1, out, 10, w, None)):
            with pytest.raises(lv.LvError) as e:
                lv.lv_kv_compact(h, *a)
            assert e.value.status == lv.LV_ERR_INVALID, a
        for a in ((sids, one, -1), (sids, one, 4097), (None, one, 1), (sids, None, 1)):
            with pytest.raises(lv.LvError) as e:
                lv.lv_session_truncate(h, *a)
            assert e.value.status == lv.LV_ERR_INVALID, a
        for w2 in (s.weights[:1], s.weights.double(), s.weights[..., ::2], s.weights.cpu(), s.weights[0]):
            with pytest.raises(ValueError):
                s.pool.select_kept(sids, one, w2)
        with pytest.raises(ValueError):
            s.pool.select_kept(sids, torch.from_numpy(one).cuda(), s.weights)
        with pytest.raises(ValueError):
            s.pool.compact(sids, one, out[:, :1])
        none = s.pool.evict_tokens(_i32([]), _i32([]), s.weights)
        assert none.shape[0] == 0 and s.pool.sync(raise_on_error=False) == 0
        _check_cut(s, [50])
    finally:
        s.close()


def test_evict_tokens_on_a_stream_and_replayed():
    """The three calls in a row on the pool's own stream; and captured, on other weights each time."""
    import torch
    side = torch.cuda.Stream()
    s = Kept([300, 120], dim=64, stream=side)
    try:
        keeps = [100, 50]
        kept = [s.choose(i, keeps[i], 2, 8) for i in range(2)]
        kv, w = s.moved(range(2), keeps, kept)
        torch.cuda.synchronize()
        got = s.pool.evict_tokens(s.sids, _i32(keeps), s.weights, first=2, last=8)
        side.synchronize()
        for i in range(2):
            assert np.array_equal(got[i, :, :, :keeps[i]].cpu().numpy(), kept[i])
        assert np.array_equal(s.kv.cpu().numpy(), kv) and np.array_equal(s.weights.cpu().numpy(), w)
        _check_cut(s, keeps)
    finally:
        s.close()
    s = Kept([300, 120], dim=64)
    try:
        sids, keeps = torch.from_numpy(s.sids).cuda(), torch.tensor([299, 119], dtype=torch.int32, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.pool.evict_tokens(sids, torch.tensor([300, 300], dtype=torch.int32, device="cuda"), s.weights, most=300)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = s.pool.evict_tokens(sids, keeps, s.weights, first=1, last=4, most=300)
        for lens in ([299, 119], [150, 119], [7, 3]):
            keeps.copy_(torch.tensor(lens, dtype=torch.int32))
            s.weights.copy_(torch.from_numpy(s.some_weights(tuple(s.weights.shape))))
            kept = [s.choose(i, lens[i], 1, 4) for i in range(2)]
            kv, w = s.moved(range(2), lens, kept)
            torch.cuda.synchronize()
            graph.replay()
            assert s.pool.sync(raise_on_error=False) == 0
            for i in range(2):
                assert np.array_equal(got[i, :, :, :lens[i]].cpu().numpy(), kept[i])
            assert np.array_equal(s.kv.cpu().numpy(), kv) and np.array_equal(s.weights.cpu().numpy(), w)
            s.total = lens
            _check_cut(s, lens)
    finally:
        s.close()


@pytest.mark.parametrize("tiers", ["LV_TIERS_EXCLUSIVE", "LV_TIERS_INCLUSIVE"])
def test_cuts_beside_appends(tiers):
    """Contexts are cut on one stream while others grow on another: every page has one owner, and its bit."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = Kept([4000, 5, 3000, 9], dim=8, heads=1, layers=1, page=8, tiers=getattr(lv, tiers), spare=6000)
    try:
        a, b = torch.cuda.Stream(), torch.cuda.Stream()
        cut, grow = (0, 2), (1, 3)
        sids = torch.from_numpy(s.sids[list(cut)].astype(np.int32)).cuda()
        lens = [torch.tensor([4000 - 40 * k, 3000 - 30 * k], dtype=torch.int32, device="cuda") for k in range(1, 60)]
        pages, count = torch.empty(64, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        for k, x in enumerate(lens):
            lv.lv_session_truncate(s.pool.handle, sids, x, 2, a)
            lv.lv_session_append(s.pool.handle, int(s.sids[grow[k % 2]]), 60, pages, count, b)
        torch.cuda.synchronize()
        assert s.pool.sync(raise_on_error=False) == 0
        ctx = s.pool.get_sessions()["ctx_tokens"]
        want = {0: 4000 - 40 * 59, 1: 5 + 60 * 30, 2: 3000 - 30 * 59, 3: 9 + 60 * 29}
        tables, hbm, _ = s.pool.tables()
        owned = np.full(len(hbm), -1, np.int64)
        for i, sid in enumerate(s.sids):
            assert ctx[sid] == want[i]
            nb = -(-want[i] // 8)
            row = tables[sid]
            assert (row[:nb] >= 0).all() and (row[nb:] == -1).all()
            assert (owned[row[:nb]] == -1).all()
            owned[row[:nb]] = (int(sid) << 16) | np.arange(nb)
        assert np.array_equal(hbm.astype(np.int64), owned)
        assert s.pool.stats()["hbm_allocated"] == (owned >= 0).sum()
        # and the bits: what is taken next is what nobody has, the lowest first
        free = np.flatnonzero(owned < 0)
        got = s.pool.append(int(s.sids[1]), 800)
        assert s.pool.sync(raise_on_error=False) == 0 and got.tolist() == free[:len(got)].tolist()
    finally:
        s.close()


def test_the_longest_lists():
    """Lists with room for 2^31 - 1 tokens, the most there may be: filled to their end, and taken by compaction."""
    import torch
    s = Kept([40, 30], heads=1, dim=8, layers=1)
    try:
        most = 2 ** 31 - 1
        kept = s.choose(1, 7, 1, 2)
        kv, w = s.moved([1], [7], [None, kept])
        got = s.pool.select_kept(s.sids[1:], _i32([7]), s.weights, first=1, last=2, most=most)
        assert s.pool.sync(raise_on_error=False) == 0 and got.shape == (1, 1, 1, most)
        assert np.array_equal(got[0, :, :, :7].cpu().numpy(), kept)
        assert int(got[0, 0, 0, 7:].max()) == int(got[0, 0, 0, 7:].min()) == -1
        lens = s.pool.compact(s.sids[1:], _i32([7]), got, s.weights)
        assert s.pool.sync(raise_on_error=False) == 0 and lens.tolist() == [7]
        assert np.array_equal(s.kv.cpu().numpy(), kv) and np.array_equal(s.weights.cpu().numpy(), w)
    finally:
        s.close()


def test_choice_of_more_sessions_than_are_ordered_by_length():
    """80 sessions, one of them long: the lists come in the sessions' order, with the long one's room in shared memory."""
    total = [17 + 31 * i % 500 for i in range(79)] + [66000]
    s = Kept(total, heads=1, dim=8, layers=1)
    try:
        keeps = [1 + t // 3 for t in total]
        got = s.pool.select_kept(s.sids, _i32(keeps), s.weights, first=2, last=3)
        assert s.pool.sync(raise_on_error=False) == 0
        _chosen(s, keeps, got.cpu().numpy(), 2, 3)
    finally:
        s.close()
