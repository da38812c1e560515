"""Serving steps on resident KV (lv_batch_plan, lv_kv_write, lv_attention) against the definitions
in 64 bits: single tokens, chunks and both, page sizes, head shapes, lengths from zero on, windows
with first tokens, work that is cut and joined, strides, and what the pages hold beside the context."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _step(*a, **kw):
    import torch
    from tests._attention import Step
    if "dtype" in kw:
        kw["dtype"] = {"bf16": torch.bfloat16, "f16": torch.float16}[kw["dtype"]]
    return Step(*a, **kw)


def _attend(s, layer=1, scale=None, lse=True, **plan):
    s.plan(**plan)
    scale = s.dim ** -0.5 if scale is None else scale
    out, z = s.batch.attention(layer, s.q, scale=scale, return_lse=True)
    assert s.pool.sync(raise_on_error=False) == 0
    return s.check(out, z, layer, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,group,dim", [(2, 4, 64), (4, 8, 128), (1, 1, 128), (3, 5, 96), (8, 16, 64), (2, 3, 8),
                                             (1, 8, 256), (2, 7, 200)])
def test_single_tokens(heads, group, dim, dtype):
    s = _step([0, 1, 15, 16, 17, 200, 1023, 3000], [1] * 8, heads=heads, group=group, dim=dim, dtype=dtype, sharp=2.0,
              pad=2)
    try:
        _attend(s)
    finally:
        s.close()


@pytest.mark.parametrize("page", [1, 2, 5, 8, 16, 24, 32, 48, 128, 256, 500])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [2, 1, 3, 2], [70, 1, 129, 0]])
def test_page_sizes(page, new):
    s = _step([31, 700, 0, 128], new, heads=2, group=8, dim=128, page=page)
    try:
        _attend(s)
    finally:
        s.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("heads,group,dim", [(2, 4, 64), (4, 8, 128), (1, 1, 128), (3, 5, 96), (1, 16, 64), (2, 7, 40),
                                             (1, 24, 128), (2, 3, 192)])
def test_chunks(heads, group, dim, dtype):
    s = _step([0, 300, 1000, 17, 127], [130, 1, 257, 64, 129], heads=heads, group=group, dim=dim, dtype=dtype, pad=3)
    try:
        _attend(s)
    finally:
        s.close()


@pytest.mark.parametrize("cached,new", [([5000], [1]), ([20000], [2]), ([9000, 10], [40, 1]), ([0], [1500]),
                                        ([300] * 40, [1] * 40), ([12000, 3, 700], [300, 90, 1])])
def test_cut_and_joined(cached, new):
    s = _step(cached, new, heads=2, group=8, dim=128, sharp=3.0)
    try:
        _attend(s)
    finally:
        s.close()


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (16, 0), (100, 1), (128, 16), (129, 130), (1000, 33),
                                          (4000, 4), (3, 700)])
@pytest.mark.parametrize("cached,new", [([0, 5, 1000, 2500], [1, 1, 1, 1]), ([0, 700, 1500], [200, 140, 1])])
def test_windows(cached, new, window, sinks):
    s = _step(cached, new, heads=2, group=4, dim=128, window=window, sinks=sinks, pad=1)
    try:
        _attend(s)
    finally:
        s.close()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("heads", [1, 4])
def test_neighbouring_long_joins(heads, new):
    """Long contexts side by side, each cut into so many pieces that they are joined in groups, of
    lengths that let a group begin with a context's last piece, where the next context begins."""
    rng = np.random.default_rng(heads)
    for n in (3, 5, 8):
        s = _step(rng.integers(9000 // heads, 60000 // heads, n).tolist(), [new] * n, heads=heads, group=8, dim=64)
        try:
            for _ in range(3):
                _attend(s)
        finally:
            s.close()


@pytest.mark.parametrize("new", [[1, 3], [70, 1, 33]])
@pytest.mark.parametrize("dim", [64, 128, 72])
@pytest.mark.parametrize("offset,gap", [(0, 0), (8, 0), (16, 16), (24, 8), (3, 5)])
def test_output_alignments(offset, gap, dim, new):
    """Outputs whose rows lie at any offset and stride; what is beside them is left alone."""
    import torch
    s = _step([40] * len(new), new, heads=2, group=4, dim=dim)
    s.plan()
    Hq = 8
    row = Hq * (dim + gap) + gap
    buf = torch.full((offset + s.rows * row + 64,), 7.0, dtype=s.dtype, device="cuda")
    out = buf[offset:].as_strided((s.rows, Hq, dim), (row, dim + gap, 1))
    assert s.batch.attention(0, s.q, out=out) is out
    assert s.pool.sync(raise_on_error=False) == 0
    s.check(out, None, 0, dim ** -0.5)
    out.fill_(7.0)
    assert (buf == 7.0).all()
    s.close()
