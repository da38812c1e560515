"""The edges of what lv_attention takes: the largest scales."""
import ctypes

import pytest

from tests._attention import Step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 40])
def test_largest_scales(new):
    """Scales are taken as long as their product with log2(e) is a 32-bit number."""
    import torch
    from paper_2606_22983_gb300 import lv
    s = Step([50], [new], heads=1, group=4, dim=64)
    try:
        s.plan()
        q, out = torch.zeros_like(s.q), torch.zeros_like(s.q)
        arg = lambda x: ctypes.byref(lv.lv_heads(data=x.data_ptr(), row_stride=256, head_stride=64, dtype=lv.LV_BF16))
        call = lambda scale: lv.lib().lv_attention(s.batch.handle, 0, arg(q), arg(out), None, scale, None)
        assert call(2.358e38) == lv.LV_OK              # every score is zero: the mean of the rows seen
        assert s.pool.sync(raise_on_error=False) == 0
        s.check(out, None, 0, 1.0, q=q)
        out.fill_(7.0)
        for scale in (2.3587e38, 3e38, 3.4e38):
            assert call(scale) == lv.LV_ERR_INVALID, scale
        assert s.pool.sync(raise_on_error=False) == 0 and (out == 7.0).all()
    finally:
        s.close()
