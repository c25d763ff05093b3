"""Counts that pass the page table's room: the keys that the table holds are seen, and no others."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_gpu_cache import FORMATS, _check, _fill, _gen, _ints, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 4), (40, 4)])
@pytest.mark.parametrize("D", [64, 192])
@pytest.mark.parametrize("pages", [1, 9, 10, 16])   # of 16 keys: rooms that end inside a tile, or with one
@pytest.mark.parametrize("cached", [1000, 2**31 - 1])
def test_cached_tokens_past_the_table(cached, pages, D, T, G, fmt, dtype):
    heads, room = 2, 16 * pages
    # the same keys as a sequence whose new tokens see none of one another
    same = _make([room], [T], heads, D, 16, fmt)
    _fill(same, [room], [0])
    for t in (same.k, same.v):   # (nothing that a key past the room could be taken for)
        t.copy_(torch.where(t.float().isnan(), 0.5, t.float()).to(t.dtype))
    c = qlin.PagedCache(**(vars(same) | dict(page_table=same.page_table[:, :pages], cached=_ints([cached]))))
    q = torch.randn(T, heads * G, D, generator=_gen(5), device="cuda").to(dtype)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = qlin.qlin_cache_attention(c, q, 0.1, lse=lse)
    assert qlin.qlin_sync_status() == 1
    bits = torch.zeros(T, T, dtype=torch.bool, device="cuda")
    _check(same, q, 0.1, bits, fmt, out, lse)


def test_values_that_are_not_finite_past_the_table():
    """The last tile's values are looked over as behind any cache: those seen come out."""
    heads, D, G, T = 1, 64, 4, 40
    same = _make([24], [T], heads, D, 8, "bf16", junk=0.5)
    _fill(same, [24], [0])
    same.v[same.page_table[0, 2].long(), 5, 0, 3] = float("inf")
    c = qlin.PagedCache(**(vars(same) | dict(page_table=same.page_table[:, :3], cached=_ints([1000]))))
    q = torch.randn(T, G, D, generator=_gen(5), device="cuda").to(torch.bfloat16)
    out = qlin.qlin_cache_attention(c, q, 0.1)
    assert qlin.qlin_sync_status() == 1
    assert (out[..., 3] == float("inf")).all() and out[..., :3].isfinite().all() and out[..., 4:].isfinite().all()
