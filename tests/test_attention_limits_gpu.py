"""The edges of what lv_attention takes: the largest scales, many query heads a KV head, infinite scores."""
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


@pytest.mark.parametrize("group", [17, 65, 100, 128, 129, 200, 256])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 32), (64, 5), (256, 16)])
@pytest.mark.parametrize("new", [[1, 1, 1], [5, 1, 0]])
def test_large_groups(group, dim, page, new):
    """Groups of more heads than a tile has rows, or than a half of one: tokens cut between tiles, halves
    of one token, queries by plain loads."""
    s = Step([0, 300, 40], new, heads=2 if group < 200 else 1, group=group, dim=dim, page=page, pad=1)
    try:
        s.plan()
        scale = dim ** -0.5
        out, lse = s.batch.attention(1, s.q, scale=scale, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        s.check(out, lse, 1, scale)
    finally:
        s.close()


@pytest.mark.parametrize("group,window", [(129, 20), (256, 0), (40, 7)])
def test_large_groups_cut_and_windowed(group, window):
    s = Step([6000, 200], [3, 7], heads=1, group=group, dim=128, window=window, sinks=3 if window else 0)
    try:
        s.plan()
        out, lse = s.batch.attention(0, s.q, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        s.check(out, lse, 0, 128 ** -0.5)
    finally:
        s.close()


@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("new", [[1, 1], [60, 1]])
def test_infinite_scores(new, page):
    """Keys whose scores are -inf weigh nothing; a score of +inf makes its rows NaN, as 1 / inf * inf is, and
    leaves other requests' rows alone."""
    import torch
    inf = float("inf")
    s = Step([200, 90], new, heads=2, group=4, dim=64, page=page)
    try:
        s.plan()
        q = s.q.clone()
        q[..., 0] = q[..., 0].abs() + 0.1

        def element(i, j):
            return s.kv[0][int(s.table[s.sids[i], j // page]), j % page, :, 0]

        hidden = [(i, j) for i in range(2) for j in (1, 17, 18, 64, 83)]
        for i, j in hidden:
            element(i, j).fill_(0.0)
        dot = s.attention64(0, 0.125, q)[3]               # magnitudes of the finite scores
        for i, j in hidden:
            element(i, j).fill_(-inf)
        want, mag, want_lse, _ = s.attention64(0, 0.125, q)
        out, lse = s.batch.attention(0, q, scale=0.125, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        score, u = dot * 2.0 ** -20 + 2.0 ** -19, 2.0 ** -8
        assert ((out.double() - want).abs() <= u * want.abs() + (1.02 * u + 4 * score[..., None]) * mag + 1e-6).all()
        assert ((lse.double() - want_lse).abs() <= 4 * score + 2.0 ** -18 * (1 + want_lse.abs())).all()
        element(0, 64).fill_(inf)
        out2, lse2 = s.batch.attention(0, q, scale=0.125, return_lse=True)
        assert s.pool.sync(raise_on_error=False) == 0
        assert torch.isnan(out2[:new[0]]).all() and not torch.isfinite(lse2[:new[0]]).any()
        assert torch.equal(out2[new[0]:], out[new[0]:]) and torch.equal(lse2[new[0]:], lse[new[0]:])
    finally:
        s.close()
