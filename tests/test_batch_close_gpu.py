"""Batches of a pool that come and go: a closed one leaves nothing behind."""
import gc
import weakref

import numpy as np
import pytest

from tests._attention import Step

pytestmark = pytest.mark.gpu


def test_closed_batches_leave_nothing():
    import torch
    from paper_2606_22983_gb300 import lv
    from paper_2606_22983_gb300.batch import KVBatch
    s = Step([20, 300], [1, 2], heads=2, group=4, dim=64)
    side = torch.cuda.Stream()
    try:
        s.plan()
        want = s.batch.attention(0, s.q)
        torch.cuda.synchronize()

        def one(rows):
            b = KVBatch(s.pool, q_heads=8, max_requests=4096, max_tokens=rows)
            b.plan(s.sids, np.array([1, 2], np.int32))
            assert torch.equal(b.attention(0, s.q), want)
            out = b.attention(0, s.q, stream=side)
            side.synchronize()
            assert torch.equal(out, want)
            tables = weakref.ref(b.tables)
            b.close()
            b.close()
            gc.collect()
            assert tables() is None
            return b

        one(5)
        torch.cuda.synchronize()
        attached, held = len(s.pool._attached), torch.cuda.memory_allocated()
        free = torch.cuda.mem_get_info()[0]
        for rows in range(5, 45):
            b = one(rows)
        torch.cuda.synchronize()
        assert len(s.pool._attached) == attached and torch.cuda.memory_allocated() <= held
        assert torch.cuda.mem_get_info()[0] >= free - (64 << 20)      # (a workspace is some 20 MiB: 40 of them)
        with pytest.raises(lv.LvError):                               # a closed batch refuses
            b.plan(s.sids, np.array([1, 2], np.int32))
        with pytest.raises(lv.LvError):
            b.attention(0, s.q)
        assert torch.equal(s.batch.attention(0, s.q), want)           # the others are as they were
        assert s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()
        assert s.batch.handle is None
