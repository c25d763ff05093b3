"""The status word keeps a wait that gave up, whatever a later call finds."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_gpu_cache import _fill, _gen, _ints, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["table", "counts", "append"])
@pytest.mark.parametrize("T,G", [(1, 4), (40, 4)])
def test_a_time_out_stays_when_tables_are_wrong(T, G, what):
    heads, D = 2, 64
    c = _make([100], [T], heads, D, 16, "bf16")
    _fill(c, [100], [T])
    q = torch.randn(T, heads * G, D, generator=_gen(1), device="cuda").to(torch.bfloat16)
    kv = q[:, :heads]
    if what == "table":
        c.page_table[0, 3] = -1
    else:
        c.cached.copy_(_ints([10**6]))

    def call():
        if what == "append":
            qlin.qlin_cache_append(c, kv, kv)
        else:
            qlin.qlin_cache_attention(c, q, 0.125)

    assert qlin.qlin_sync_status() == 0
    call()
    assert qlin.qlin_sync_status() == 1
    qlin.qlin_selftest_bounded_wait(1_000_000)   # nothing completes this wait of 1 ms
    call()
    assert qlin.qlin_sync_status() == 5
    call()
    qlin.qlin_selftest_bounded_wait(1_000_000)
    assert qlin.qlin_sync_status() == 5
    assert qlin.qlin_sync_status() == 0
