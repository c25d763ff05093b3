"""Outputs of the cache calls whose rows would lie over one another are refused (no GPU needed); rows
that interleave are not."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_serving_args import A16, INVALID, WORKSPACE, _append, _attention, _cache, lib  # noqa: F401

# (tokens, heads, token stride, head stride) in heads of 128, and whether rows meet
MEET = [(4, 4, 1, 1), (4, 4, 1, 2), (2, 4, 3, 1), (4, 2, 1, 3), (4, 4, 2, 3), (3, 4, 3, 2), (4, 4, -1, 1), (4, 4, 2, -4)]
APART = [(4, 4, 4, 1), (4, 4, 1, 4), (2, 2, 2, 3), (2, 4, 7, 2), (4, 2, 2, 9), (1, 4, 0, 1), (3, 2, 2, 1)]


def _meet(T, H, ts, hs):
    rows = [t * ts + h * hs for t in range(T) for h in range(H)]
    return len(set(rows)) < len(rows)


def test_the_lists():
    assert all(_meet(*c) for c in MEET) and not any(_meet(*c) for c in APART)


def _refused(lib, T, H, ts, hs):
    assert lib.qlin_cache_attention(_cache(), _attention(tokens=T, q_heads=H, out_token_stride=ts, out_head_stride=hs),
                                    A16, 1 << 30, None) == INVALID
    assert lib.qlin_cache_append(_cache(), _append(tokens=T, q_heads=H, q_out_token_stride=ts, q_out_head_stride=hs),
                                 None) == INVALID


@pytest.mark.parametrize("T,H,ts,hs", MEET)
def test_rows_that_meet_are_refused(lib, T, H, ts, hs):  # noqa: F811
    _refused(lib, T, H, 128 * ts, 128 * hs)


@pytest.mark.parametrize("T,H,ts,hs", [(2, 4, 128, 200), (2, 4, 200, 136), (2, 4, 136, -200), (2, 4, 776, 256),
                                       (2**20, 4, 128, 2**27 - 64)])
def test_rows_that_meet_in_part_are_refused(lib, T, H, ts, hs):  # noqa: F811
    _refused(lib, T, H, ts, hs)


@pytest.mark.parametrize("ts,hs,meet", [(2**62, 2**62, True), (-2**63, 2**63 - 8, True), (2**63 - 8, 2**63 - 8, True),
                                        (2**62, 2**60, False), (-2**63, 2**60, False)])
def test_strides_of_any_size(lib, ts, hs, meet):  # noqa: F811
    status = lib.qlin_cache_attention(_cache(), _attention(tokens=4, q_heads=4, out_token_stride=ts, out_head_stride=hs),
                                      A16, 0, None)
    assert status == (INVALID if meet else WORKSPACE)   # (apart: the next check, of the workspace, is met)


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,ts,hs", [c for c in APART if c[2] >= 0])
def test_rows_that_interleave(T, H, ts, hs):
    D = 64
    i32 = dict(dtype=torch.int32, device="cuda")
    kv = torch.randn(2, 16, 1, D, device="cuda").to(torch.bfloat16)
    c = qlin.PagedCache(kv, kv.flip(0).contiguous(), torch.tensor([[1, 0]], **i32), torch.tensor([20], **i32),
                        torch.tensor([0, T], **i32))
    q = torch.randn(T, H, D, device="cuda").to(torch.bfloat16)
    want = qlin.qlin_cache_attention(c, q, 0.125)
    buf = torch.full((64 * D,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf.as_strided((T, H, D), (ts * D, hs * D, 1))
    qlin.qlin_cache_attention(c, q, 0.125, out=out)
    assert torch.equal(out, want) and (buf == 7).sum() >= (64 - T * H) * D
    buf.fill_(7.0)
    k = torch.zeros(T, 1, D, dtype=torch.bfloat16, device="cuda")
    qlin.qlin_cache_append(c, k, k, qlin.rope_plan(D), q=q, q_out=out)
    assert torch.equal(out, qlin.qlin_cache_append(c, k, k, qlin.rope_plan(D), q=q))
    assert qlin.qlin_sync_status() == 0
