"""Waits inside the attention kernels that run out: whichever role's it was, the call ends, the device
reports LV_ERR_TIMEOUT, and a step planned anew gives the bits of one that nothing disturbed."""
import pytest

from tests._attention import Step

pytestmark = pytest.mark.gpu

COPIES, PRODUCTS = 1, 2
CASES = [(COPIES, [300, 40], [1, 1]), (COPIES, [30000], [1]), (COPIES, [300, 40], [40, 3]), (COPIES, [9000], [200]),
         (PRODUCTS, [100, 40], [16, 3]), (PRODUCTS, [9000], [200])]


def _run_out(s, what, layer=0):
    """An attention whose waits run out, and its status."""
    from paper_2606_22983_gb300 import lv
    lv.lv_selftest_attention(s.batch.handle, what, 20_000)
    s.batch.attention(layer, s.q)
    st = s.pool.sync(raise_on_error=False)
    lv.lv_selftest_attention(s.batch.handle, lv.LV_HOLD_NONE)
    return st


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("what,cached,new", CASES)
def test_a_wait_that_runs_out(what, cached, new, dim):
    import torch
    from paper_2606_22983_gb300 import lv
    s = Step(cached, new, heads=2, group=8, dim=dim, pad=1)
    try:
        s.plan()
        want = s.batch.attention(0, s.q, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        for _ in range(2):
            s.plan()
            assert _run_out(s, what) == lv.LV_ERR_TIMEOUT
            s.pool.clear_error()
            s.plan()
            again = s.batch.attention(0, s.q, return_lse=True)
            assert s.pool.sync(raise_on_error=False) == 0
            assert all(torch.equal(a, b) for a, b in zip(want, again))
    finally:
        s.close()


def test_selftest_refusals():
    from paper_2606_22983_gb300 import lv
    s = Step([3], [1], heads=1, group=1, dim=8)
    try:
        h, call = s.batch.handle, lv.lib().lv_selftest_attention
        for args in ((None, 0, 0), (h, -1, 20_000), (h, 3, 20_000), (h, 1, 999), (h, 2, 1_000_001), (h, 1, -1)):
            assert call(*args) == lv.LV_ERR_INVALID, args
        s.plan()
        s.check(s.batch.attention(0, s.q), None, 0, 8 ** -0.5)
        assert s.pool.sync(raise_on_error=False) == 0
    finally:
        s.close()


@pytest.mark.parametrize("what,cached,new", [c for c in CASES if c[0] == COPIES])
def test_a_step_with_a_timeout_is_planned_again(what, cached, new):
    """Its counts of arrived pieces are not those of a fresh step: later calls refuse it."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = Step(cached, new, heads=2, group=8, dim=128, pad=1)
    try:
        s.plan()
        want = s.batch.attention(1, s.q, return_lse=True)
        assert _run_out(s, what) == lv.LV_ERR_TIMEOUT
        s.pool.clear_error()
        out = torch.full_like(s.q, 7.0)
        s.batch.attention(1, s.q, out=out)
        st = s.pool.stats()
        assert st["error"] == lv.LV_ERR_STATE and st["error_detail"] == -1
        assert (out == 7.0).all()
        s.pool.clear_error()
        s.plan()
        again = s.batch.attention(1, s.q, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        assert all(torch.equal(a, b) for a, b in zip(want, again))
    finally:
        s.close()
