"""Serving steps on a stream other than the current one: memory that a launch uses, or that it makes its
results in, is not given to others before it has run; and batches on streams of their own."""
import numpy as np
import pytest

from tests._attention import Step
from tests.test_batch_gpu import _plan_by_hand

pytestmark = pytest.mark.gpu

LATE = 40_000_000          # cycles that a stream is kept busy, some 20 ms


@pytest.fixture(params=["given", "the pool's"])
def busy(request):
    """A step and a function that keeps its stream busy; sized so that a dropped tensor's memory is the
    next one's of its size."""
    import torch
    s = Step([100, 30], [1500, 4], heads=2, group=4, dim=64, pad=2)
    side = torch.cuda.Stream()
    kw = {"stream": side}
    if request.param == "the pool's":
        s.pool.stream, kw = side, {}
    s.plan(**kw)
    torch.cuda.synchronize()

    def late():
        with torch.cuda.stream(side):
            torch.cuda._sleep(LATE)

    yield s, side, kw, late
    torch.cuda.synchronize()
    assert s.pool.sync(raise_on_error=False) == 0
    s.close()


def test_dropped_results(busy):
    import torch
    s, side, kw, late = busy
    for _ in range(3):
        late()
        out, lse = s.batch.attention(0, s.q, return_lse=True, **kw)
        del out, lse
        mine = torch.full_like(s.q, 7.0), torch.full((s.rows, 8), 7.0, device="cuda")
        side.synchronize()
        torch.cuda.synchronize()
        assert all((x == 7.0).all() for x in mine)


def test_results_beside_the_current_streams_work(busy):
    """The current stream still reads a tensor that the program has dropped."""
    import torch
    s, side, kw, late = busy
    for _ in range(3):
        old, kept = torch.full_like(s.q, 3.0), torch.empty_like(s.q)
        torch.cuda.synchronize()
        torch.cuda._sleep(LATE)
        kept.copy_(old)
        del old
        out = s.batch.attention(0, s.q, **kw)
        side.synchronize()
        torch.cuda.synchronize()
        assert (kept == 3.0).all()
        s.check(out, None, 0, 0.125)


def test_dropped_arguments(busy):
    import torch
    s, side, kw, late = busy
    for _ in range(3):
        q = s.q.clone()
        k, v = (torch.randn((s.rows, 2, 64), device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        kv = s.kv.clone()
        slots = _plan_by_hand(s)[4]
        for i, slot in enumerate(slots):
            if slot >= 0:
                for j, y in enumerate((k, v)):
                    kv[j].view(-1, 2, 64)[slot] = y[i].to(s.dtype)
        torch.cuda.synchronize()
        late()
        s.batch.write(0, k, v, **kw)
        out = s.batch.attention(0, q, **kw)
        del q, k, v
        torch.full_like(s.q, 7.0), [torch.full((s.rows, 2, 64), 7.0, device="cuda") for _ in range(2)]
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(s.kv.view(torch.int16), kv.view(torch.int16))
        s.check(out, None, 0, 0.125)


def test_dropped_ids_and_lengths(busy):
    import torch
    s, side, kw, late = busy
    for _ in range(3):
        sids, lens = (torch.from_numpy(np.asarray(x, np.int32)).cuda() for x in (s.sids, s.new))
        torch.cuda.synchronize()
        late()
        s.batch.plan(sids, lens, num_tokens=s.rows, max_len=max(s.new), **kw)
        del sids, lens
        torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        side.synchronize()
        torch.cuda.synchronize()
        assert np.array_equal(s.batch.slots[:s.rows].cpu().numpy(), _plan_by_hand(s)[4])


def test_batches_on_streams_of_their_own():
    """Two batches of one pool at once, each kernel beside the other and beside itself."""
    import torch
    from paper_2606_22983_gb300.batch import KVBatch
    for new in ([1, 2, 1, 1], [300, 1, 77, 130]):
        s = Step([3000, 100, 9000, 0], [300, 2, 77, 130], heads=2, group=8, dim=128)
        try:
            steps = []
            for lens in ([1, 2, 1, 1], new):
                rows = sum(lens)
                b = KVBatch(s.pool, q_heads=16, max_requests=4, max_tokens=rows)
                q = torch.randn((rows, 16, 128), device="cuda").to(s.dtype)
                lens = np.asarray(lens, np.int32)
                b.plan(s.sids, lens)
                steps.append((b, q, lens, b.attention(0, q), torch.cuda.Stream()))
            torch.cuda.synchronize()
            outs = []
            for _ in range(10):
                for b, q, lens, _, stream in steps:
                    with torch.cuda.stream(stream):
                        b.plan(s.sids, lens)
                        outs.append(b.attention(0, q))
            torch.cuda.synchronize()
            assert s.pool.sync(raise_on_error=False) == 0
            for i, out in enumerate(outs):
                assert torch.equal(out, steps[i % 2][3])
        finally:
            s.close()
