"""A block's step for fewer tokens than it has rows gives what it gives without the steps before it."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_gpu_block import _make, _paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", [("fp8", torch.bfloat16), ("nvfp4", torch.float8_e4m3fn)])
@pytest.mark.parametrize("M,full,fewer", [(4, [1, 1, 1, 1], [1, 1]), (100, [70, 30], [20, 33])])
@pytest.mark.parametrize("bad", [False, True])
def test_a_step_does_not_depend_on_the_one_before(fmt, dtype, M, full, fewer, bad):
    b, x, pos = _make(fmt, M)
    fresh, _, _ = _make(fmt, M)
    before, after, again = _paged(full, [40] * len(full), dtype), *(_paged(fewer, [33, 5], dtype) for _ in "ab")
    if dtype is torch.bfloat16:
        before.v.mul_(100.0)   # (the step before has values far above)
    else:
        before.v_scale = before.v_scale * 100.0
    if bad:
        before.v_scale, before.v = ((before.v_scale, torch.full_like(before.v, float("inf")))
                                    if dtype is torch.bfloat16 else (before.v_scale * float("nan"), before.v))
    b.step(x, pos, before)
    n = sum(fewer)
    y = b.step(x, pos, after)[:n].clone()
    assert not b.attended[n:].any()
    want = fresh.step(x, pos, again)[:n]
    assert qlin.qlin_sync_status() == 0
    assert torch.isfinite(y.float()).all() and torch.equal(y, want)
    s = torch.cuda.Stream()   # on a stream of its own, and replayed
    s.wait_stream(torch.cuda.current_stream())
    b.step(x, pos, before, stream=s)
    other = b.step(x, pos, after, stream=s)
    s.synchronize()
    assert torch.equal(other[:n], y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(x, pos, before)
        b.step(x, pos, after)
    for _ in range(2):
        b.y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.y[:n], y)
