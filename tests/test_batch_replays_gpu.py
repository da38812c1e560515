"""Captured writes and attention, replayed under later plans: the rows of the plan that the device made
last, and nothing but a report where the capture does not fit it."""
import numpy as np
import pytest

from tests._attention import Step
from tests.test_batch_gpu import _plan_by_hand

pytestmark = pytest.mark.gpu

FEW, MANY = [1, 2, 0, 2], [40, 1, 70, 9]      # new tokens (of 8 heads a KV head): each attention kernel's


class Captured:
    """A step's write and attention in a graph, over tensors of `rows` rows."""

    def __init__(self, s, rows, planned_before):
        import torch
        s.new, s.rows = list(planned_before), rows
        s.cached = [t - m for t, m in zip(s.total, s.new)]
        self.s, self.rows, Hq = s, rows, s.heads * s.group
        self.k, self.v = (torch.randn((rows, s.heads, s.dim), device="cuda") for _ in range(2))
        self.q = torch.randn((rows, Hq, s.dim), device="cuda").to(s.dtype)
        self.out = torch.empty_like(self.q)
        s.plan()
        s.batch.write(1, self.k, self.v)
        s.batch.attention(1, self.q, out=self.out)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            s.batch.write(1, self.k, self.v)
            s.batch.attention(1, self.q, out=self.out)

    def plan(self, new, num_tokens, **kw):
        s = self.s
        s.new, s.rows = list(new), num_tokens
        s.cached = [t - m for t, m in zip(s.total, new)]
        s.plan(**kw)
        assert s.pool.sync(raise_on_error=False) == 0

    def replay(self):
        """New values, a replay, and the K and V arrays as they should be after it."""
        import torch
        s = self.s
        self.k.normal_(), self.v.normal_(), self.q.normal_(), self.out.fill_(7.0)
        want = s.kv.clone()
        if s.rows <= self.rows:
            for i, slot in enumerate(_plan_by_hand(s)[4]):
                if slot >= 0:
                    for kv, y in enumerate((self.k, self.v)):
                        want[2 + kv].view(-1, s.heads, s.dim)[slot] = y[i].to(s.dtype)
        self.graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s.kv.view(torch.int16), want.view(torch.int16))

    def check(self):
        """The output is the attention of the plan's rows, and zeros in the other rows."""
        s = self.s
        assert s.pool.sync(raise_on_error=False) == 0
        s.rows = self.rows                    # (rows past the plan's are of no request)
        s.check(self.out, None, 1, s.dim ** -0.5, q=self.q)
        assert (self.out[sum(s.new):] == 0).all()

    def refused(self):
        from paper_2606_22983_gb300 import lv
        st = self.s.pool.stats()
        assert st["error"] == lv.LV_ERR_STATE and st["error_detail"] == -1
        self.s.pool.clear_error()
        assert (self.out == 7.0).all()


def _captured(planned_before, rows):
    s = Step([300, 40, 90, 200], MANY, heads=2, group=8, dim=64, max_tokens=256)
    return s, Captured(s, rows, planned_before)


@pytest.mark.parametrize("before,after", [(FEW, [1, 1, 0, 1]), (FEW, [0, 0, 0, 0]), (MANY, [17, 0, 5, 1]),
                                          (MANY, [3, 40, 60, 16])])
def test_a_plan_of_fewer_rows(before, after):
    """Rows past the later plan's are neither written nor answered, whatever the plan before left there."""
    s, c = _captured(before, sum(before) + 2)
    try:
        for num_tokens in (sum(after), sum(after) + 1, c.rows):
            c.plan(before, c.rows)            # (slots in every row of the earlier plan's requests)
            c.plan(after, num_tokens, max_len=max(before))
            c.replay()
            c.check()
    finally:
        s.close()


@pytest.mark.parametrize("before,after", [(FEW, MANY), (MANY, [1, 1, 2, 1])])
def test_a_plan_for_the_other_kernel(before, after):
    rows = sum(MANY) + 2
    s, c = _captured(before, rows)
    try:
        own = list(s.new)
        c.plan(after, sum(after), max_len=max(after))
        c.replay()                            # (the write takes any plan of as many rows)
        c.refused()
        c.plan(own, rows, max_len=max(own))
        c.replay()
        c.check()
    finally:
        s.close()


@pytest.mark.parametrize("before,after", [(FEW, [2, 2, 2, 2]), ([40, 1, 20, 3], MANY)])
def test_a_plan_of_more_rows(before, after):
    s, c = _captured(before, sum(before))
    try:
        c.plan(after, sum(after))
        c.replay()                            # nothing is written either
        c.refused()
        c.plan(before, sum(before))
        c.replay()
        c.check()
    finally:
        s.close()


@pytest.mark.parametrize("steps", [[[1, 1, 1, 1], [0, 2, 1, 2], [2, 2, 2, 2]], [MANY, [5, 60, 0, 33], [0, 0, 0, 1]]])
def test_a_captured_plan(steps):
    """The plan in the graph too: its ids and lengths are read when it is replayed."""
    import torch
    rows = max(map(sum, steps)) + 1
    s = Step([300, 40, 90, 200], [max(x) for x in zip(*steps)], heads=2, group=8, dim=64, max_tokens=256)
    try:
        most = max(map(max, steps))
        sids, lens = torch.from_numpy(s.sids).cuda(), torch.zeros(4, dtype=torch.int32, device="cuda")
        k, v = (torch.randn((rows, 2, 64), device="cuda") for _ in range(2))
        q = torch.randn((rows, 16, 64), device="cuda").to(s.dtype)
        out = torch.empty_like(q)

        def step():
            s.batch.plan(sids, lens, num_tokens=rows, max_len=most)
            s.batch.write(0, k, v)
            s.batch.attention(0, q, out=out)

        step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for new in steps:
            lens.copy_(torch.tensor(new, dtype=torch.int32))
            s.new, s.rows = list(new), rows
            s.cached = [t - m for t, m in zip(s.total, new)]
            k.normal_(), v.normal_(), q.normal_()
            g.replay()
            torch.cuda.synchronize()
            assert s.pool.sync(raise_on_error=False) == 0
            want = _plan_by_hand(s)
            assert np.array_equal(s.batch.slots[:rows].cpu().numpy(), want[4])
            assert np.array_equal(s.batch.positions[:rows].cpu().numpy(), want[3])
            s.check(out, None, 0, 64 ** -0.5, q=q)
            assert (out[sum(new):] == 0).all()
    finally:
        s.close()


@pytest.mark.parametrize("which", ["sids", "lens", "firsts"])
def test_a_captured_plan_takes_no_pageable_memory(which):
    """A replay would read it again, when the program has given it back."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = Step([30, 7], [1, 1], heads=1, group=2, dim=8)
    try:
        host = {"sids": s.sids, "lens": np.array([1, 1], np.int32), "firsts": np.array([-1, -1], np.int32)}
        dev = {n: torch.from_numpy(x).cuda() for n, x in host.items()}
        s.batch.plan(*(dev[n] for n in ("sids", "lens", "firsts")), num_tokens=2, max_len=1)
        out = torch.zeros_like(s.q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            with pytest.raises(lv.LvError) as e:
                s.batch.plan(*({**dev, which: host[which]}[n] for n in ("sids", "lens", "firsts")),
                             num_tokens=2, max_len=1)
            assert e.value.status == lv.LV_ERR_INVALID
            s.batch.plan(*(dev[n] for n in ("sids", "lens", "firsts")), num_tokens=2, max_len=1)
            s.batch.attention(0, s.q, out=out)
        g.replay()
        torch.cuda.synchronize()
        assert s.pool.sync(raise_on_error=False) == 0
        s.check(out, None, 0, 8 ** -0.5)
    finally:
        s.close()
