"""Attention behind shared prefixes: every row against the definition in 64 bits, the plan's arrays, what the
calls refuse and report, and what must not change a result."""
import numpy as np
import pytest

from tests._attention import Step
from tests._shared import SharedStep

pytestmark = pytest.mark.gpu


def _run(s, layer=1, scale=None, **kw):
    scale = s.dim ** -0.5 if scale is None else scale
    s.plan(**kw)
    out, lse = s.batch.attention(layer, s.q, scale=scale, return_lse=True)
    assert s.pool.sync(raise_on_error=False) == 0
    s.check(out, lse, layer, scale)
    return out, lse


SHAPES = {
    "one": dict(cached=[5], new=[1], of=[0], prefix=[1]),
    "unit": dict(cached=[0, 1], new=[1, 1], of=[0, 0], prefix=[128]),
    "tokens": dict(cached=[30, 200, 0, 77], new=[1, 1, 1, 1], of=[0, 0, 0, 0], prefix=[1001]),
    # prefixes of which only a part is continued, requests without one or without tokens between them
    "parts": dict(cached=[9, 0, 300, 16, 40, 2], new=[3, 2, 0, 1, 4, 1], of=[0, 0, 0, -1, 1, 1], prefix=[700, 129],
                  plens=[333, 0]),
    # one prefix in two runs, and another between them
    "runs": dict(cached=[64, 3, 150, 8, 31], new=[1, 2, 5, 1, 1], of=[0, 0, 1, 0, -1], prefix=[260, 515]),
    "chunks": dict(cached=[0, 100, 17], new=[150, 33, 260], of=[0, 0, -1], prefix=[391]),
    "many": dict(cached=[4 * i % 90 for i in range(300)], new=[1] * 300, of=[i // 120 for i in range(300)],
                 prefix=[90, 47, 512]),
    # a long prefix in many pieces
    "long": dict(cached=[20, 40], new=[1, 1], of=[0, 0], prefix=[30011]),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(shape, dtype):
    import torch
    s = SharedStep(**SHAPES[shape], heads=2, group=4, dim=64, pad=3, dtype=getattr(torch, dtype))
    try:
        _run(s)
    finally:
        s.close()


# (12 tokens of 8 rows at most: the kernel for few rows; pages of 5 and dims above 128 have no other)
@pytest.mark.parametrize("heads,group,dim,page", [(1, 1, 128, 16), (4, 8, 128, 16), (2, 7, 96, 32), (1, 16, 64, 64), (3, 5, 80, 8),
                                                  (1, 200, 64, 16), (2, 3, 256, 16), (2, 4, 64, 5), (1, 2, 8, 1)])
def test_shapes(heads, group, dim, page):
    for new in ([1, 1, 1, 1, 1], [40, 1, 7, 1, 2]):
        s = SharedStep([33, 250, 0, 64, 5], new, [0, 0, 0, 1, 1], [300, 70], heads=heads, group=group, dim=dim, page=page)
        try:
            _run(s)
        finally:
            s.close()


@pytest.mark.parametrize("sharp", [8.0, 60.0])
def test_far_maxima(sharp):
    """Scores far apart: one side's weights vanish beside the other's."""
    s = SharedStep([60, 3, 200], [2, 1, 1], [0, 0, 0], [450], heads=2, group=4, dim=64, sharp=sharp)
    try:
        _run(s)
    finally:
        s.close()


def test_small_pieces_of_few_rows():
    """One row of one head and a prefix in many pieces: the kernel for few rows, joined in two steps."""
    s = SharedStep([2000], [1], [0], [40007], heads=1, group=4, dim=64)
    try:
        _run(s)
    finally:
        s.close()


@pytest.mark.parametrize("where", ["numpy", "device", "pinned"])
def test_plan(where):
    import torch
    conv = {"numpy": lambda x: x, "device": lambda x: torch.from_numpy(x).cuda(),
            "pinned": lambda x: torch.from_numpy(x).pin_memory()}[where]
    s = SharedStep([9, 0, 300, 16], [3, 2, 0, 1], [0, 0, 1, -1], [700, 129], plens=[333, 129], heads=1, group=2, dim=8, pad=2)
    try:
        s.plan(conv)
        assert s.pool.sync(raise_on_error=False) == 0
        b = s.batch
        assert b.row_starts[:5].tolist() == [0, 3, 5, 5, 6]
        assert b.kv_lens[:4].tolist() == [12, 2, 300, 17]                  # their own
        assert b.positions[:8].tolist() == [342, 343, 344, 333, 334, 16, -1, -1]
        for i in range(4):
            nb = -(-s.total[i] // s.page)
            assert b.tables[i, :nb].tolist() == s.table[s.sids[i], :nb].tolist() and (b.tables[i, nb:] == -1).all()
        own = [s.table[s.sids[i], p // 16] * 16 + p % 16 for i, p in ((0, 9), (0, 10), (0, 11), (1, 0), (1, 1), (3, 16))]
        assert b.slots[:8].tolist() == own + [-1, -1]
    finally:
        s.close()


def test_same_as_one_context():
    """A prefix of whole pages and a session behind it give what one session of all their tokens gives."""
    import torch
    s = SharedStep([40, 100], [1, 6], [0, 0], [512], heads=2, group=4, dim=64)
    try:
        out, lse = _run(s)
        t = Step([552, 612], [1, 6], heads=2, group=4, dim=64)
        try:
            for i in range(2):
                for kv in range(4):
                    x = Step.rows_of(s, s.requests, kv % 2, kv // 2), Step.rows_of(s, i, kv % 2, kv // 2)
                    x = torch.cat(x).to(t.dtype)
                    j = torch.arange(len(x), device="cuda")
                    t.kv[kv][torch.from_numpy(t.table[t.sids[i]].astype(np.int64)).cuda()[j // 16], j % 16] = x
            t.plan()
            same, lse2 = t.batch.attention(1, s.q, scale=0.125, return_lse=True)
            assert t.pool.sync(raise_on_error=False) == 0
            assert torch.equal(t.batch.positions[:7], s.batch.positions[:7])
            # either is off by at most what check() allows; here they differ by the order of sums
            assert ((out.double() - same.double()).abs() <= 2.0 ** -6 * (1 + same.double().abs())).all()
            assert ((lse - lse2).abs() <= 2.0 ** -16 * (1 + lse2.abs())).all()
        finally:
            t.close()
    finally:
        s.close()


@pytest.mark.parametrize("what", ["sid", "longer", "negative", "absent", "own"])
def test_requests_left_out(what):
    """A request whose prefix breaks a rule is reported and left out; the others go on, in two runs."""
    from paper_2606_22983_gb300 import lv
    absent = {(4, 2)} if what == "absent" else ()
    s = SharedStep([20, 50, 7], [3, 2, 4], [0, 1, 0], [100, 60], plens=[100, 60], heads=2, group=4, dim=64, absent=absent)
    try:
        n = 3
        pre = np.array([s.psid(i) for i in range(n)], np.int32)
        lens = np.array([100, 60, 100], np.int32)
        sids = s.sids[:n].copy()
        if what == "sid":
            pre[1] = s.pool.S
        elif what == "longer":
            lens[1] = 61
        elif what == "negative":
            lens[1] = -1
        elif what == "own":
            sids[1] = -1
        s.batch.plan(sids, np.array(s.new[:n], np.int32), prefixes=pre, prefix_lens=lens)
        out, lse = s.batch.attention(0, s.q, scale=0.125, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == (lv.LV_ERR_STATE if what == "absent" else lv.LV_ERR_BOUNDS)
        assert s.pool.stats()["error_detail"] == 1
        assert s.batch.kv_lens[:n].tolist() == [23, 0, 11] and (s.batch.positions[3:5] == -1).all()
        want, mag, want_lse, _ = s.attention64(0, 0.125)
        want[3:5], mag[3:5], want_lse[3:5] = 0, 0, -float("inf")
        assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * mag + 1e-5).all()
        assert (out[3:5] == 0).all() and (lse[3:5] == -float("inf")).all()
    finally:
        s.close()


def test_a_part_that_is_resident():
    """Of a prefix only the blocks of the continued tokens have to be in HBM."""
    s = SharedStep([20], [1], [0], [100], plens=[40], heads=2, group=4, dim=64, absent={(1, 4), (1, 6)})
    try:
        _run(s)
    finally:
        s.close()


def test_refusals():
    from paper_2606_22983_gb300 import lv
    from paper_2606_22983_gb300.batch import KVBatch
    s = SharedStep([20, 5], [1, 2], [0, 0], [50], heads=2, group=4, dim=64)
    try:
        make = lambda **kw: KVBatch(s.pool, **{**dict(q_heads=8, max_requests=4, max_tokens=8), **kw})
        for kw in (dict(window=5, prefix_rows=3), dict(prefix_rows=9), dict(prefix_rows=-1)):
            with pytest.raises(lv.LvError) as e:
                make(**kw)
            assert e.value.status == lv.LV_ERR_INVALID
        small, none = make(prefix_rows=2), make()
        sids, one, pre = s.sids[:2], np.array([1, 2], np.int32), np.full(2, s.psid(0), np.int32)
        for b in (small, none):
            with pytest.raises(lv.LvError) as e:
                b.plan(sids, one, prefixes=pre)
            assert e.value.status == lv.LV_ERR_INVALID
        with pytest.raises(lv.LvError) as e:
            lv.lv_batch_share(small.handle, 2)              # it has the room
        assert e.value.status == lv.LV_ERR_INVALID
        small.plan(sids[:1], one[:1], prefixes=pre[:1])
        assert s.pool.sync(raise_on_error=False) == 0
        with pytest.raises(ValueError):
            small.plan(sids[:1], one[:1], prefixes=pre)
        with pytest.raises(ValueError):
            small.plan(sids[:1], one[:1], prefix_lens=one[:1])
        with pytest.raises(lv.LvError):
            lv.lv_batch_plan_shared(small.handle, sids[:1], None, one[:1], None, None, 1, 1, 1, 0)
        # no request: as a plan without prefixes
        small.plan(sids[:0], one[:0], prefixes=pre[:0], num_tokens=2)
        assert (small.attention(0, s.q[:2]) == 0).all() and s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()


def test_plans_of_either_kind_in_turn():
    """The same batch with prefixes, without, and with again."""
    import torch
    s = SharedStep([20, 50, 7], [3, 2, 4], [0, -1, 0], [600], heads=2, group=4, dim=64)
    try:
        first, _ = _run(s)
        s.batch.plan(s.sids[:3], np.array(s.new[:3], np.int32))
        out = s.batch.attention(1, s.q, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == 0
        assert torch.equal(out[3:5], first[3:5]) and not torch.equal(out[:3], first[:3])
        again, _ = _run(s)
        assert torch.equal(first, again)
    finally:
        s.close()


def test_replayed():
    """A captured plan, write and attention on lengths that change; a step without prefixes is refused there."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = SharedStep([20, 300, 7], [2, 2, 2], [0, 0, 0], [600], plens=[600], heads=2, group=4, dim=64)
    try:
        n, dev = 3, lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        sids, lens, pre, plens = dev(s.sids[:n].tolist()), dev([2, 2, 2]), dev([s.psid(0)] * 3), dev([600] * 3)
        out = torch.empty_like(s.q)
        go = lambda: (s.batch.plan(sids, lens, prefixes=pre, prefix_lens=plens, num_tokens=6, max_len=2),
                      s.batch.attention(1, s.q, out=out, scale=0.125))
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            go()
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                go()
        for of, part in (([0, 0, 0], 600), ([0, -1, 0], 129), ([-1, -1, -1], 5), ([0, 0, 0], 599)):
            s.of, s.plens = of, [part]
            pre.copy_(dev([s.psid(i) for i in range(n)]))
            plens.fill_(part)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert s.pool.sync(raise_on_error=False) == 0
            s.check(out, None, 1, 0.125)
        alone = torch.cuda.CUDAGraph()
        with torch.cuda.graph(alone, stream=side):
            s.batch.attention(1, s.q, out=out, scale=0.125)
        s.batch.plan(sids, lens, num_tokens=6, max_len=2)
        out.fill_(3.0)
        alone.replay()
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and (out == 3.0).all()
        assert s.pool.stats()["error_detail"] == -1
        s.pool.clear_error()
        other = torch.cuda.CUDAGraph()
        with torch.cuda.graph(other, stream=side):
            s.batch.attention(1, s.q, out=out, scale=0.125)
        other.replay()
        assert s.pool.sync(raise_on_error=False) == 0 and not (out == 3.0).any()
        go()
        out.fill_(3.0)
        other.replay()
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and (out == 3.0).all()
    finally:
        s.close()


@pytest.mark.parametrize("new", [[1], [30]])
def test_waits_that_run_out(new):
    """A wait inside the pass over the prefixes ends with a report; the step is refused until planned again."""
    from paper_2606_22983_gb300 import lv
    s = SharedStep([200], new, [0], [3000], heads=2, group=4, dim=64)
    try:
        s.plan()
        lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_COPIES, 2000)
        s.batch.attention(0, s.q)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_TIMEOUT
        s.pool.clear_error()
        lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_NONE)
        s.batch.attention(0, s.q)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE
        s.pool.clear_error()
        _run(s)
    finally:
        s.close()


def test_strides_and_streams():
    import torch
    s = SharedStep([20, 300, 7], [2, 40, 2], [0, 0, 0], [600], heads=2, group=4, dim=64)
    try:
        want, lse = _run(s)
        wide = torch.zeros((s.rows, 8, 3 * 64 + 1), dtype=s.dtype, device="cuda")
        q, out = wide[..., 65:129], torch.zeros((s.rows, 16, 64), dtype=s.dtype, device="cuda")[:, ::2]
        q.copy_(s.q)
        s.batch.attention(1, q, out=out, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == 0 and torch.equal(out, want)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        s.plan(stream=side)
        got, l2 = s.batch.attention(1, s.q, scale=0.125, return_lse=True, stream=side)
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(l2, lse)
    finally:
        s.close()


@pytest.mark.parametrize("group", [5, 7, 12, 100])
@pytest.mark.parametrize("kind", ["alone", "behind"])
def test_the_same_each_time(group, kind):
    """Groups whose rows do not fill the tensor core's: what shared memory held before has no say in the result."""
    import torch
    cached, new = [128, 512, 3, 40], [700, 900, 60, 333]
    kw = dict(heads=2, group=group, dim=64)
    s = SharedStep(cached, new, [0, 0, -1, 0], [900], **kw) if kind == "behind" else Step(cached, new, **kw)
    try:
        s.plan()
        far = 30 * s.q                                     # (what an attention between leaves there)
        want, want_lse = s.batch.attention(1, s.q, scale=0.125, return_lse=True)
        for k in range(8):
            s.batch.attention(1, far if k & 1 else s.q.flip(0), scale=0.125)
            out, lse = s.batch.attention(1, s.q, scale=0.125, return_lse=True)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()
