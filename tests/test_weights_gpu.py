"""Attention weights added up for the cached tokens: against the definition in 64 bits, what the call refuses and
reports, and a run of it with the attention before it and the choice of tokens after it."""
import numpy as np
import pytest

from tests._attention import Step
from tests._shared import SharedStep

pytestmark = pytest.mark.gpu


def _weights(s, seed=3, slack=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn((s.pool.S, s.heads, s.pool.max_blocks * s.page + slack), generator=g, device="cuda").exp()
    return w * 0.01


def _want(s, w, lse, layer, scale, last=0, skip=(), q=None):
    """The weights afterwards in 64 bits, and how far 32 bits may be off: each weight by its score's error (the
    sum of |q k| times 2^-19, what head_dim products lose in 32 bits, and twice 2^-20 for the exponent's
    roundings, of which lse's conversion to powers of two takes |lse| 2^-23), and by one rounding for each addition."""
    import torch
    q = (s.q if q is None else q).double()
    out, tol = w.double().clone(), torch.zeros_like(w, dtype=torch.float64)
    adds = torch.ones_like(out)
    at = 0
    prefixed = isinstance(s, SharedStep)
    for i in range(s.requests if prefixed else s.n):
        m = s.new[i]
        before = s.before(i) if prefixed else 0
        k, hidden = s.rows_of(i, 0, layer), ~s.seen(i)
        lo = max(0, m - last) if last else 0
        for h in range(s.heads * s.group if m > lo else 0):
            kk, x, z = k[:, h // s.group], q[at + lo:at + m, h], lse[at + lo:at + m, h].double()[:, None]
            y = torch.exp((x @ kk.T) * scale - z)
            off = (x.abs() @ kk.abs().T) * scale * 2.0 ** -19 + 2.0 ** -19 + z.abs() * 2.0 ** -23
            live = ~hidden[lo:] & torch.isfinite(z)
            y, off = torch.where(live, y, 0.0), torch.where(live, y * off, 0.0)
            n = live.sum(0).double()
            for what, part in (("own", slice(before, None)), ("prefix", slice(0, before))):
                if (what == "prefix" and not before) or (what, i) in skip:
                    continue
                sid = s.sids[i] if what == "own" else s.psid(i)
                span = (int(sid), h // s.group, slice(0, y[:, part].shape[1]))
                out[span] += y[:, part].sum(0)
                tol[span] += off[:, part].sum(0)
                adds[span] += n[part]
        at += m
    return out, tol + adds * 2.0 ** -24 * out.abs() + 1e-30


def _check(got, want, tol, before):
    import torch
    assert (got.double() - want).abs().le(tol).all(), ((got.double() - want).abs() / tol).max().item()
    untouched = want == before.double()
    assert torch.equal(got[untouched], before[untouched])


def _run(s, layer=1, scale=None, last=0, slack=0, **kw):
    scale = s.dim ** -0.5 if scale is None else scale
    s.plan(**kw)
    _, lse = s.batch.attention(layer, s.q, scale=scale, return_lse=True)
    w = _weights(s, slack=slack)
    before = w.clone()
    s.batch.add_weights(layer, s.q, lse, w, last=last, scale=scale)
    assert s.pool.sync(raise_on_error=False) == 0
    _check(w, *_want(s, before, lse, layer, scale, last), before)
    again = before.clone()
    s.batch.add_weights(layer, s.q, lse, again, last=last, scale=scale)
    assert (again == w).all()                     # bit for bit
    return w, lse, before


STEPS = {
    "one": dict(cached=[0], new=[1]),
    "keys": dict(cached=[127, 128, 255, 256, 63], new=[1, 1, 1, 1, 1]),
    "tokens": dict(cached=[30, 2000, 0, 777], new=[1, 1, 1, 2]),
    "mixed": dict(cached=[9, 0, 300, 16, 40], new=[3, 200, 0, 1, 70]),
    "prompt": dict(cached=[0], new=[700]),
    "chunk": dict(cached=[1500], new=[130]),
    "many": dict(cached=[(7 * i) % 400 for i in range(300)], new=[1 + i % 3 for i in range(300)]),
}


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("step", STEPS)
def test_weights(step, dtype):
    import torch
    s = Step(**STEPS[step], heads=2, group=4, dim=64, pad=3, dtype=getattr(torch, dtype))
    try:
        _run(s)
    finally:
        s.close()


@pytest.mark.parametrize("heads,group,dim,page", [(1, 1, 128, 16), (4, 8, 128, 16), (2, 7, 96, 32), (1, 16, 64, 64), (3, 5, 80, 8),
                                                  (1, 200, 64, 16), (2, 3, 256, 16), (2, 4, 64, 5), (1, 2, 8, 1), (2, 48, 72, 24)])
def test_shapes(heads, group, dim, page):
    s = Step([33, 250, 0, 64, 515], [1, 40, 7, 0, 2], heads=heads, group=group, dim=dim, page=page)
    try:
        _run(s, slack=1)
    finally:
        s.close()


@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 4), (129, 130), (1000, 0), (16, 300)])
@pytest.mark.parametrize("last", [0, 5])
def test_windows(window, sinks, last):
    """Under a window only what a row sees has a weight; blocks that none sees may be elsewhere."""
    absent = {(1, 5)} if window == 100 else ()
    s = Step([20, 700, 0, 130], [3, 1, 400, 40], heads=2, group=4, dim=64, window=window, sinks=sinks, absent=absent)
    try:
        _run(s, last=last)
    finally:
        s.close()


@pytest.mark.parametrize("last", [1, 16, 64, 1000])
def test_last_rows(last):
    s = Step([20, 700, 5], [300, 1, 33], heads=2, group=4, dim=128)
    try:
        _run(s, last=last)
    finally:
        s.close()


@pytest.mark.parametrize("last", [0, 2])
@pytest.mark.parametrize("shape", [
    dict(cached=[30, 200, 0, 77], new=[1, 1, 1, 1], of=[0, 0, 0, 0], prefix=[1001]),
    dict(cached=[9, 0, 300, 16, 40, 2], new=[3, 2, 0, 1, 4, 1], of=[0, 0, 0, -1, 1, 1], prefix=[700, 129], plens=[333, 0]),
    dict(cached=[0, 100, 17, 5], new=[150, 33, 260, 1], of=[0, 0, -1, 1], prefix=[391, 128])])
def test_behind_prefixes(shape, last):
    s = SharedStep(**shape, heads=2, group=4, dim=64, pad=1)
    try:
        _run(s, last=last)
    finally:
        s.close()


@pytest.mark.parametrize("sharp", [10.0, 60.0])
def test_far_scores(sharp):
    s = Step([900, 40], [1, 30], heads=2, group=4, dim=64, sharp=sharp)
    try:
        _run(s)
    finally:
        s.close()


def test_rows_without_a_sum_and_odd_values():
    """A row whose lse is -inf has no weights, one of +inf zeros; a NaN stays with the keys of its row."""
    import torch
    s = Step([100, 60, 30], [1, 2, 1], heads=1, group=4, dim=64)
    try:
        s.plan()
        _, lse = s.batch.attention(0, s.q, scale=0.125, return_lse=True)
        odd = lse.clone()
        odd[0, 1], odd[1], odd[3, 2] = -float("inf"), float("inf"), float("nan")
        w = _weights(s)
        before = w.clone()
        s.batch.add_weights(0, s.q, odd, w, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == 0
        assert torch.isnan(w[s.sids[2], 0, :31]).all() and not torch.isnan(w[s.sids[2], 0, 31:]).any()
        w[s.sids[2]] = before[s.sids[2]]
        odd[3] = -float("inf")
        _check(w, *_want(s, before, odd, 0, 0.125), before)
        # a NaN key is its own token's alone, and rows that are nobody's have no effect
        page = s.table[s.sids[0], 2]
        s.kv[0, page, 3, 0, 5] = float("nan")
        s.kv[0, page, 4, 0, 5] = float("inf")
        w = before.clone()
        s.batch.add_weights(0, s.q, lse, w, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == 0
        row = w[s.sids[0], 0]
        assert torch.isnan(row[35]) and not torch.isfinite(row[36])
        row[35:37] = before[s.sids[0], 0, 35:37]
        s.kv[0, page, 3:5, 0, 5] = 0
        want, tol = _want(s, before, lse, 0, 0.125)
        want[s.sids[0], 0, 35:37], tol[s.sids[0], 0, 35:37] = before[s.sids[0], 0, 35:37].double(), 1e-30
        _check(w, want, tol, before)
    finally:
        s.close()


def test_left_out():
    """Sessions that come twice, and contexts that the weights have no room for."""
    from paper_2606_22983_gb300 import lv
    s = Step([200, 90, 40], [1, 2, 1], heads=2, group=4, dim=64)
    try:
        s.plan()
        _, lse = s.batch.attention(0, s.q, scale=0.125, return_lse=True)
        w = _weights(s)
        before = w.clone()
        s.batch.add_weights(0, s.q, lse, w[..., :100], scale=0.125)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_BOUNDS and s.pool.stats()["error_detail"] == 0
        s.pool.clear_error()
        _check(w, *_want(s, before, lse, 0, 0.125, skip={("own", 0)}), before)
        sids = s.sids.copy()
        sids[2] = sids[0]
        s.batch.plan(sids, np.array([1, 2, 1], np.int32))
        _, lse = s.batch.attention(0, s.q, scale=0.125, return_lse=True)
        w = before.clone()
        s.batch.add_weights(0, s.q, lse, w, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_DOUBLE_MAP and s.pool.stats()["error_detail"] == 2
        s.pool.clear_error()
        _check(w, *_want(s, before, lse, 0, 0.125, skip={("own", 2)}), before)
    finally:
        s.close()


def test_a_prefix_in_two_runs():
    from paper_2606_22983_gb300 import lv
    s = SharedStep([64, 3, 150, 8], [1, 2, 5, 1], [0, 0, 1, 0], [260, 515], heads=2, group=4, dim=64)
    try:
        s.plan()
        _, lse = s.batch.attention(0, s.q, scale=0.125, return_lse=True)
        w = _weights(s)
        before = w.clone()
        s.batch.add_weights(0, s.q, lse, w, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_DOUBLE_MAP and s.pool.stats()["error_detail"] == 3
        s.pool.clear_error()
        _check(w, *_want(s, before, lse, 0, 0.125, skip={("prefix", 3)}), before)
    finally:
        s.close()


def test_refusals():
    import torch
    from paper_2606_22983_gb300 import lv
    s = Step([200, 90], [1, 2], heads=2, group=4, dim=64)
    try:
        w, lse = _weights(s), torch.zeros((3, 8), device="cuda")
        q = s.batch._put(lv.lv_heads(), s.q, 8, "q")
        arg = s.pool._put_weights(lv.lv_weights(), w, False)
        h = s.batch.handle
        with pytest.raises(lv.LvError) as e:                     # not planned
            lv.lv_attention_weights(h, 0, q, lse, arg, 0, 1.0, 0)
        assert e.value.status == lv.LV_ERR_INVALID
        s.plan()
        wrong = lv.lv_heads(data=q.data, row_stride=q.row_stride, head_stride=q.head_stride, dtype=lv.LV_F16)
        host = lv.lv_weights(data=np.zeros(4, np.float32).ctypes.data, tokens=1)
        for a in ((2, q, lse, arg, 0, 1.0), (-1, q, lse, arg, 0, 1.0), (0, q, lse, arg, -1, 1.0), (0, q, None, arg, 0, 1.0),
                  (0, q, lse, arg, 0, 0.0), (0, q, lse, arg, 0, float("nan")), (0, q, lse, arg, 0, 3e38), (0, wrong, lse, arg, 0, 1.0),
                  (0, q, lse, host, 0, 1.0), (0, q, lse.cpu(), arg, 0, 1.0), (0, q, lse.data_ptr() + 2, arg, 0, 1.0)):
            with pytest.raises(lv.LvError) as e:
                lv.lv_attention_weights(h, *a, 0)
            assert e.value.status == lv.LV_ERR_INVALID, a
        for a in ((s.q[:2], lse, w), (s.q, lse[:2], w), (s.q, lse.double(), w), (s.q, lse[:, ::2], w), (s.q, lse, w[:1]),
                  (s.q, lse, w.half()), (s.q, lse.T.contiguous().T, w), (s.q, lse, w[None])):
            with pytest.raises(ValueError):
                s.batch.add_weights(0, *a)
        assert torch.equal(w, _weights(s)) and s.pool.sync(raise_on_error=False) == 0
        # a step without rows; one whose attention ran out of a wait
        s.batch.plan(s.sids[:0], s.sids[:0])
        s.batch.add_weights(0, s.q[:0], lse[:0], w)
        s.plan()
        lv.lv_selftest_attention(h, lv.LV_HOLD_COPIES, 2000)
        _, lse = s.batch.attention(0, s.q, return_lse=True)
        lv.lv_selftest_attention(h, lv.LV_HOLD_NONE)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_TIMEOUT
        s.pool.clear_error()
        s.batch.add_weights(0, s.q, lse, w)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and s.pool.stats()["error_detail"] == -1
        assert torch.equal(w, _weights(s))
    finally:
        s.close()


def test_strides_and_streams():
    import torch
    s = Step([20, 300, 7], [2, 40, 2], heads=2, group=4, dim=64)
    try:
        want, lse, before = _run(s)
        wide = torch.zeros((s.rows, 8, 3 * 64 + 1), dtype=s.dtype, device="cuda")
        q = wide[..., 65:129]
        q.copy_(s.q)
        w = torch.zeros((s.heads, s.pool.S, before.shape[2] + 9), device="cuda").transpose(0, 1)[..., 4:]
        w[..., :before.shape[2]] = before
        s.batch.add_weights(1, q, lse, w, scale=0.125)
        assert s.pool.sync(raise_on_error=False) == 0
        assert torch.equal(w[..., :before.shape[2]], want) and (w[..., before.shape[2]:] == 0).all()
        side = torch.cuda.Stream()
        w = before.clone()
        torch.cuda.synchronize()
        s.batch.add_weights(1, s.q, lse, w, scale=0.125, stream=side)
        side.synchronize()
        assert torch.equal(w, want)
    finally:
        s.close()


def test_replayed():
    """Captured with the attention before it: each replay adds the step's weights that is planned then."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = Step([200, 900, 30], [1, 1, 1], heads=2, group=4, dim=64, max_tokens=9)
    try:
        w, side = _weights(s), torch.cuda.Stream()
        go = lambda: s.batch.attention(0, s.q, scale=0.125, return_lse=True)
        s.plan()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _, lse = go()
            s.batch.add_weights(0, s.q, lse, w, scale=0.125)
        before = w.clone()
        for sids, new in (([0, 1, 2], [1, 1, 1]), ([1, 2], [2, 1]), ([2], [1])):
            s.batch.plan(s.sids[sids], np.array(new, np.int32), num_tokens=3, max_len=1 if max(new) == 1 else 2)
            graph.replay()
            assert s.pool.sync(raise_on_error=False) == 0
            t = type("T", (), dict(requests=0, n=len(sids), new=new, heads=2, group=4, q=s.q, sids=s.sids[sids],
                                   rows_of=lambda self, i, kv, layer: s.rows_of(sids[i], kv, layer),
                                   seen=lambda self, i: torch.arange(s.total[sids[i]], device="cuda")[None] <=
                                   torch.arange(s.total[sids[i]] - new[i], s.total[sids[i]], device="cuda")[:, None]))()
            _check(w, *_want(t, before, lse, 0, 0.125), before)
            before = w.clone()
        big = torch.randn((9, 8, 64), device="cuda").to(s.dtype)
        s.batch.plan(s.sids, np.array([3, 3, 3], np.int32), np.array([0, 0, 0], np.int32))      # more rows than captured
        s.batch.attention(0, big)
        assert s.pool.sync(raise_on_error=False) == 0
        graph.replay()
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and torch.equal(w, before)
    finally:
        s.close()


def test_a_session_cut_by_its_weights():
    """Steps that add up weights, the eviction of tokens by them, and the steps after it, in which
    attention sees the kept tokens and no others."""
    import torch
    s = Step([190, 333], [10, 7], heads=2, group=4, dim=64)
    try:
        w = torch.zeros((2, s.pool.S, 2, s.pool.max_blocks * 16), device="cuda")
        s.plan()
        for layer in range(2):
            _, lse = s.batch.attention(layer, s.q, return_lse=True)
            s.batch.add_weights(layer, s.q, lse, w[layer], last=4)
        keeps = np.array([60, 75], np.int32)
        old = [[s.rows_of(i, kv, layer) for kv in range(2) for layer in range(2)] for i in range(2)]
        kept = s.pool.evict_tokens(s.sids, keeps, w, first=4, last=12)
        assert s.pool.sync(raise_on_error=False) == 0
        for i in range(2):
            n, c = keeps[i], s.total[i]
            assert (kept[i, :, :, :4].cpu() == torch.arange(4)).all()
            assert (kept[i, :, :, n - 12:n].cpu() == torch.arange(c - 12, c)).all()
            for k, x in enumerate(old[i]):
                kv, layer = divmod(k, 2)
                s.total[i] = c
                new = Step.rows_of(s, i, kv, layer)[:n]
                for h in range(2):
                    assert torch.equal(new[:, h], x[kept[i, layer, h, :n].long(), h])
            assert (w[:, s.sids[i], :, n:] == 0).all() and (w[:, s.sids[i], :, :4] > 0).all()
        # two more tokens of each
        s.table = None
        for i in range(2):
            s.pool.append(int(s.sids[i]), 2)
        s.table = s.pool.tables()[0].copy()
        s.cached, s.new = [int(x) for x in keeps], [2, 2]
        s.total, s.rows = [a + 2 for a in s.cached], 4
        s.batch.plan(s.sids, np.array(s.new, np.int32))
        x = torch.randn((4, 4, 64), generator=s.gen, device="cuda").to(s.dtype)
        for layer in range(2):
            s.batch.write(layer, x[:, :2], x[:, 2:])
        q = s.q[:4]
        s.q = q
        for layer in range(2):
            before = w[layer].clone()
            out, lse = s.batch.attention(layer, q, scale=0.125, return_lse=True)
            s.check(out, lse, layer, 0.125)
            s.batch.add_weights(layer, q, lse, w[layer], scale=0.125)
            assert s.pool.sync(raise_on_error=False) == 0
            _check(w[layer], *_want(s, before, lse, layer, 0.125), before)
    finally:
        s.close()


@pytest.mark.parametrize("what", ["LV_HOLD_COPIES", "LV_HOLD_PRODUCTS"])
@pytest.mark.parametrize("new", [[1, 1], [300, 1]])
def test_waits_that_run_out(new, what):
    """A wait inside the kernel ends with a report; the step is refused until it is planned again."""
    from paper_2606_22983_gb300 import lv
    s = Step([2000, 700], new, heads=2, group=4, dim=64)
    try:
        s.plan()
        _, lse = s.batch.attention(0, s.q, return_lse=True)
        w = _weights(s)
        before = w.clone()
        lv.lv_selftest_attention(s.batch.handle, getattr(lv, what), 2000)
        s.batch.add_weights(0, s.q, lse, w)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_TIMEOUT
        s.pool.clear_error()
        lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_NONE)
        w.copy_(before)
        s.batch.add_weights(0, s.q, lse, w)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and (w == before).all()
        s.pool.clear_error()
        _run(s)
    finally:
        s.close()


CUT = {
    "prompt": dict(cached=[0], new=[3000], heads=1, group=8, dim=64),
    "chunks": dict(cached=[5000, 40, 0], new=[700, 1, 2100], heads=2, group=4, dim=128, dtype="float16"),
    "short": dict(cached=[100], new=[2500], heads=1, group=48, dim=64, page=8),
    "tail": dict(cached=[0, 300], new=[2600, 900], heads=1, group=16, dim=64, last=500),
    "window": dict(cached=[0, 20], new=[2300, 1700], heads=2, group=7, dim=64, window=600, sinks=3),
    "beside": dict(cached=[(97 * i) % 1500 for i in range(200)] + [0], new=[1] * 200 + [1500], heads=1, group=16, dim=64),
}


@pytest.mark.parametrize("step", CUT)
def test_cut_units(step):
    """Keys that many rows see, shared out by rows; the sums are the same bit for bit each time."""
    import torch
    c = dict(CUT[step])
    last = c.pop("last", 0)
    s = Step(c.pop("cached"), c.pop("new"), **{**c, "dtype": getattr(torch, c.get("dtype", "bfloat16"))})
    try:
        w, lse, before = _run(s, last=last)
        for _ in range(3):
            again = before.clone()
            s.batch.add_weights(1, s.q, lse, again, last=last, scale=s.dim ** -0.5)
            s.batch.attention(1, s.q, scale=s.dim ** -0.5)      # (it counts and joins in the same memory)
            assert torch.equal(again, w)
    finally:
        s.close()


@pytest.mark.parametrize("last", [0, 300])
def test_cut_prefixes(last):
    s = SharedStep(cached=[0, 100, 17, 5], new=[500, 433, 860, 1], of=[0, 0, 0, 1], prefix=[391, 128], heads=1, group=16, dim=64)
    try:
        _run(s, last=last)
    finally:
        s.close()


def test_cut_units_after_a_wait_that_ran_out():
    """Pieces that came before a wait ran out are not counted in the next step."""
    from paper_2606_22983_gb300 import lv
    s = Step([0], [2500], heads=1, group=16, dim=64)
    try:
        s.plan()
        _, lse = s.batch.attention(0, s.q, return_lse=True)
        for what in (lv.LV_HOLD_COPIES, lv.LV_HOLD_PRODUCTS):
            lv.lv_selftest_attention(s.batch.handle, what, 2000)
            s.batch.add_weights(0, s.q, lse, _weights(s))
            assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_TIMEOUT
            s.pool.clear_error()
            lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_NONE)
            _run(s)
    finally:
        s.close()


def test_replayed_with_other_lengths():
    """A captured call takes a step of shorter or longer requests than the one before its capture: units that it does
    not cut, and cuts where there are none, give the weights all the same."""
    import torch
    s = Step([0, 40], [1200, 3], heads=1, group=16, dim=64)
    try:
        side, lse = torch.cuda.Stream(), torch.empty((s.rows, 16), device="cuda")
        steps = {"long": (np.array([1200, 3], np.int32), 1200), "short": (np.array([2, 3], np.int32), 3)}
        graphs, w = {}, torch.zeros_like(_weights(s))

        def plan(name):
            new, most = steps[name]
            s.batch.plan(s.sids, new, num_tokens=s.rows, max_len=most)
            lse.copy_(s.batch.attention(0, s.q, return_lse=True)[1])

        for name in steps:
            plan(name)
            torch.cuda.synchronize()
            graphs[name] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[name], stream=side):
                s.batch.add_weights(0, s.q, lse, w)
        for name in ("long", "short", "long"):
            plan(name)
            want = torch.zeros_like(w)
            s.batch.add_weights(0, s.q, lse, want)
            for captured, graph in graphs.items():
                w.zero_()
                graph.replay()
                assert s.pool.sync(raise_on_error=False) == 0
                if captured == name or name == "short":
                    assert torch.equal(w, want)
                else:      # (the same products' sums, added up in another order: a few roundings of 2^-24, as all are
                    # positive and what an addition loses is kept)
                    assert (w - want).abs().le(2.0 ** -20 * want).all()
    finally:
        s.close()


@pytest.mark.parametrize("new", [[1, 1], [300, 1]])
def test_after_a_wait_that_ran_out_over_a_prefix(new):
    """The attention has left no sums then: nothing is added until the step is planned again."""
    from paper_2606_22983_gb300 import lv
    s = SharedStep([200, 30], new, [0, 0], [3000], heads=2, group=4, dim=64)
    try:
        s.plan()
        lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_COPIES, 2000)
        _, lse = s.batch.attention(0, s.q, return_lse=True)
        lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_NONE)
        assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_TIMEOUT
        s.pool.clear_error()
        lse.zero_()
        w = _weights(s)
        before = w.clone()
        for _ in range(2):
            s.batch.add_weights(0, s.q, lse, w)
            assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and s.pool.stats()["error_detail"] == -1
            s.pool.clear_error()
            assert (w == before).all()
            s.batch.attention(0, s.q)
            assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE
            s.pool.clear_error()
        _run(s)
    finally:
        s.close()


@pytest.mark.parametrize("captured", ["prefix", "none", "long", "short"])
def test_replayed_behind_an_attention_that_is_refused(captured):
    """Attention and weights in one graph, replayed after a plan whose attention is another: the attention leaves the sums
    of the step before, and nothing is added; after a plan of its own kind the graph works again, as calls outside it do."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = SharedStep([200, 900], [300, 1], [0, 0], [600], heads=2, group=4, dim=64)
    try:
        sids = s.sids[:2]
        new = np.array([300, 1], np.int32)

        def plan(kind):
            if kind == "prefix":
                s.plan()
            else:
                s.batch.plan(sids, new if kind != "short" else np.array([2, 1], np.int32), num_tokens=s.rows,
                             max_len=2 if kind == "short" else 300)

        def both():
            _, lse = s.batch.attention(0, s.q, scale=0.125, return_lse=True)
            s.batch.add_weights(0, s.q, lse, w, scale=0.125)

        w, side = _weights(s), torch.cuda.Stream()
        before = w.clone()
        plan(captured)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
        graph.replay()
        assert s.pool.sync(raise_on_error=False) == 0
        want = w.clone()
        assert not torch.equal(want, before)
        for other in {"prefix": ("long", "short"), "none": ("prefix", "short"), "long": ("short",), "short": ("long", "prefix")}[captured]:
            plan(other)
            w.copy_(before)
            graph.replay()
            assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE and s.pool.stats()["error_detail"] == -1
            s.pool.clear_error()
            assert torch.equal(w, before)
            both()                               # (an attention that runs is followed by its weights)
            assert s.pool.sync(raise_on_error=False) == 0 and not torch.equal(w, before)
            graph.replay()
            assert s.pool.sync(raise_on_error=False) == lv.LV_ERR_STATE
            s.pool.clear_error()
            plan(captured)                       # a new plan's sums may come from elsewhere
            w.copy_(before)
            graph.replay()
            assert s.pool.sync(raise_on_error=False) == 0 and torch.equal(w, want)
    finally:
        s.close()


@pytest.mark.parametrize("dim", [64, 256])
def test_captured_before_there_was_room_for_prefixes(dim):
    """A call captured on a batch that gets its room for prefixes later works on a step behind one all the same."""
    import torch
    from paper_2606_22983_gb300 import lv
    from paper_2606_22983_gb300.batch import KVBatch
    s = SharedStep([64, 3, 150, 8], [1, 2, 5, 1], [0, 0, 1, -1], [260, 515], heads=2, group=4, dim=dim)
    try:
        s.batch.close()
        s.batch = KVBatch(s.pool, q_heads=8, max_requests=4, max_tokens=s.rows, dtype=s.dtype)
        s.batch.plan(s.sids[:4], np.asarray(s.new[:4], np.int32))
        lse, w = torch.empty((s.rows, 8), device="cuda"), _weights(s)
        before, side = w.clone(), torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.batch.add_weights(0, s.q, lse, w, scale=0.125)
        lv.lv_batch_share(s.batch.handle, s.rows)
        s.plan()
        lse.copy_(s.batch.attention(0, s.q, scale=0.125, return_lse=True)[1])
        graph.replay()
        assert s.pool.sync(raise_on_error=False) == 0
        _check(w, *_want(s, before, lse, 0, 0.125), before)
    finally:
        s.close()


@pytest.mark.parametrize("shape", [dict(cached=[100], new=[300], heads=2, group=4, dim=64),
                                   dict(cached=[100], new=[300], heads=2, group=4, dim=256),
                                   dict(cached=[0], new=[2500], heads=1, group=16, dim=64)])
def test_infinite_weights(shape):
    """A row whose exponentials exceed 32 bits makes the weights of the keys it sees infinite, and no others."""
    import torch
    s = Step(**shape)
    try:
        s.plan()
        scale = s.dim ** -0.5
        _, lse = s.batch.attention(0, s.q, scale=scale, return_lse=True)
        before = _weights(s)
        want, w = before.clone(), before.clone()
        s.batch.add_weights(0, s.q, lse, want, scale=scale)
        lse[20, 1] = -1e5                       # (scores are far above -1e4)
        s.batch.add_weights(0, s.q, lse, w, scale=scale)
        assert s.pool.sync(raise_on_error=False) == 0
        sees = s.cached[0] + 21
        row, other = w[s.sids[0], 0], want[s.sids[0], 0]
        assert (row[:sees] == float("inf")).all()
        assert torch.equal(row[sees:], other[sees:]) and torch.equal(w[s.sids[0], 1:], want[s.sids[0], 1:])
    finally:
        s.close()


HALVES = {
    # contexts that end in the first half of their last 256 keys, beside longer ones: units of one half and of two
    "one size": dict(cached=[300] * 40, new=[70] * 40, heads=2, group=16, dim=64),
    "sizes": dict(cached=[(97 * i) % 700 for i in range(60)], new=[1 + (41 * i) % 120 for i in range(60)], heads=4, group=8, dim=128),
    "long rows": dict(cached=[512, 255, 88, 144, 0, 1110, 274, 1716, 511, 2636, 58, 3775, 299], new=[4, 2, 6, 3, 10, 8, 75, 7, 8, 11, 24, 5, 40],
                      heads=4, group=100, dim=128, page=24),
}


@pytest.mark.parametrize("step", HALVES)
def test_units_of_one_half_beside_two(step):
    """A half without keys leaves its sums at once, however far the other is."""
    import torch
    s = Step(**HALVES[step])
    try:
        w, lse, before = _run(s)
        for _ in range(20):
            again = before.clone()
            s.batch.add_weights(1, s.q, lse, again, scale=s.dim ** -0.5)
            assert torch.equal(again, w)
        assert s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()


def test_prefixes_of_one_half():
    """Three prefixes of 128 tokens in front of contexts of all lengths, the last rows of each."""
    import torch
    cached = [2476, 3568, 8, 1670, 0, 832, 0, 127, 115, 244, 3670, 0, 127, 216, 0, 256, 177, 2530, 1024, 0, 210, 127, 277, 1024, 256,
              256, 127, 7, 2383, 1, 319, 1, 0, 12, 0, 163, 3810, 128, 1024, 121]
    new = [4, 4, 1307, 1, 1, 1, 1, 1, 1427, 1445, 1, 880, 0, 1, 0, 1, 1035, 1275, 2, 1352, 507, 1, 1, 1, 1, 4, 1, 1, 1, 1, 3, 1244,
           898, 354, 617, 0, 1066, 0, 1057, 1]
    s = SharedStep(cached, new, [-1] * 7 + [0] * 11 + [1] * 14 + [2] * 8, [128, 128, 128], heads=2, group=16, dim=96, page=32)
    try:
        w, lse, before = _run(s, last=3)
        for _ in range(20):
            again = before.clone()
            s.batch.add_weights(1, s.q, lse, again, last=3, scale=s.dim ** -0.5)
            assert torch.equal(again, w)
        assert s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()


@pytest.mark.parametrize("dim,page", [(64, 16), (256, 16), (64, 5)])
def test_the_most_sessions(dim, page):
    """4095 requests of one token each behind the 4096th session's: a segment for each, in steps of one run and of 2000."""
    import torch
    from paper_2606_22983_gb300.batch import KVBatch
    from paper_2606_22983_gb300.pool import KVPool
    S, n, P, G = 4096, 4095, 300, 2
    blocks = -(-P // page)
    pages = n + blocks
    gen = torch.Generator(device="cuda").manual_seed(dim)
    kv = torch.randn((2, pages, page, 1, dim), generator=gen, device="cuda").to(torch.bfloat16)
    pool = KVPool(layers=1, kv_heads=1, head_dim=dim, page_tokens=page, max_sessions=S, max_blocks=blocks, hbm_pages=pages,
                  hbm_budget_pages=pages, host_pages=0, kv=kv.view(torch.uint8).view(2, pages, page * dim * 2))
    try:
        table = np.full((S, blocks), -1, np.int32)
        table[:n, 0], table[n] = np.arange(n), np.arange(n, pages)
        ctx = np.ones(S, np.int32)
        ctx[n] = P
        pool.import_placement(table, ctx)
        batch = KVBatch(pool, q_heads=G, max_requests=S, max_tokens=n, prefix_rows=n)
        q = torch.randn((n, G, dim), generator=gen, device="cuda").to(torch.bfloat16)
        sids = np.random.default_rng(1).permutation(n).astype(np.int32)
        own = kv[0, :n, 0, 0].double()[torch.from_numpy(sids).long().cuda()]
        before = kv[0, n:, :, 0].reshape(-1, dim)[:P].double()
        for many in (n, 2000):
            batch.plan(sids, np.ones(n, np.int32), prefixes=np.where(np.arange(n) < many, n, -1).astype(np.int32))
            _, lse = batch.attention(0, q, scale=0.1, return_lse=True)
            w = torch.zeros((S, 1, blocks * page), device="cuda")
            batch.add_weights(0, q, lse, w, scale=0.1)
            assert pool.sync(raise_on_error=False) == 0
            x, z = q.double(), lse.double()[:, :, None]
            dot = torch.einsum("rgd,kd->rgk", x.abs(), before.abs()).amax() * 0.1
            mine = torch.exp(torch.einsum("rgd,rd->rg", x, own)[:, :, None] * 0.1 - z)[:, :, 0].sum(1)
            pre = torch.exp(torch.einsum("rgd,kd->rgk", x[:many], before) * 0.1 - z[:many]).sum((0, 1))
            # (as in _want, with the largest sum of |q k| for all, and its additions of 2 and of 2 * many)
            tol = (dot + (x.abs().sum(2).amax() * own.abs().amax()) * 0.1) * 2.0 ** -19 + 2.0 ** -18 + z.abs().amax() * 2.0 ** -23
            got = w[:, 0].double()
            assert ((got[torch.from_numpy(sids).long().cuda(), 0] - mine).abs() <= tol * mine).all()
            assert ((got[n, :P] - pre).abs() <= (tol + 2 * many * 2.0 ** -24) * pre).all()
            assert (got[:n, 1:] == 0).all() and (got[n, P:] == 0).all()
    finally:
        pool.close()
