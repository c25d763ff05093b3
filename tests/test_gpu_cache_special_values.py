"""Attention over a paged cache where queries, keys, values or scales are NaN or infinite: the
formula's NaN comes out of every row that they reach, whether its keys lie in one CTA or are split
among several, and the other rows keep their bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_gpu_cache import FORMATS, UNIT, _check, _fill, _gen, _make, _slots

pytestmark = pytest.mark.gpu

HEADS, D = 2, 64
# new tokens, query heads of a KV head (few rows and many), cached tokens (one CTA's keys and many CTAs')
FORMS = [(1, 4, 20), (1, 4, 1000), (1, 4, 20000), (40, 4, 20), (40, 4, 3000), (40, 4, 20000)]


def _call(c, q, scale=0.125):
    lse = torch.full(q.shape[:2], 5.0, device="cuda")
    out = qlin.qlin_cache_attention(c, q, scale, lse=lse)
    assert qlin.qlin_sync_status() == 0
    return out, lse


def _largest_value(c, where):
    v = c.v[where].double().nan_to_num(0)
    return v.abs().max().item() * (1.0 if c.v_scale is None else c.v_scale.item())


def _setup(T, G, have, fmt, dtype):
    c = _make([have], [T], HEADS, D, 16, fmt)
    _fill(c, [have], [T])
    return c, torch.randn(T, HEADS * G, D, generator=_gen(5), device="cuda").to(dtype)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("T,G,have", FORMS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_a_query_that_is_not_finite_gives_nan(bad, T, G, have, fmt, dtype):
    c, q = _setup(T, G, have, fmt, dtype)
    good, good_lse = _call(c, q)
    q[T - 1, 1, 7] = bad   # (an infinity times keys of both signs: scores of both infinities)
    out, lse = _call(c, q)
    assert out[T - 1, 1].isnan().all() and lse[T - 1, 1].isnan()
    rest = torch.ones(T, HEADS * G, dtype=torch.bool, device="cuda")
    rest[T - 1, 1] = False
    assert torch.equal(out[rest], good[rest]) and torch.equal(lse[rest], good_lse[rest])


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("T,G,have", FORMS)
def test_a_nan_among_keys_of_little_weight(T, G, have, fmt, dtype):
    """The first half's keys are zero, the others' scores lie 300 powers of two above: what is NaN in
    the first half has a weight that fp32 does not hold, and still reaches every row."""
    c, q = _setup(T, G, have, fmt, dtype)
    q.fill_(1.0)
    where = _slots(c, 0, have + T)
    c.k[where] = torch.zeros((), device="cuda").to(c.k.dtype)
    high = tuple(i[have // 2:] for i in where)
    c.k[high] = torch.full((), 4.0 if c.k_scale is None else 4.0 / c.k_scale.item(), device="cuda").to(c.k.dtype)
    scale = 300 / (4 * D) * math.log(2)   # (E4M3: 4 / k_scale = 298.7 is 288, 289 powers of two)
    good, good_lse = _call(c, q, scale)
    assert good.isfinite().all() and good_lse.isfinite().all()
    page, slot = (int(i[have // 4]) for i in where)
    nan = torch.full((), math.nan, device="cuda").to(c.v.dtype)
    for t in (c.v, c.k):
        old = t[page, slot, 1].clone()
        t[page, slot, 1, 3] = nan
        out, lse = _call(c, q, scale)
        assert torch.equal(out[:, :G], good[:, :G]) and torch.equal(lse[:, :G], good_lse[:, :G])
        if t is c.v:
            assert out[:, G:, 3].isnan().all() and torch.equal(lse, good_lse)
            others = [d for d in range(D) if d != 3]
            off = (out.double() - good.double())[..., others].abs()
            # Of a tile that holds new tokens the few-row kernel adds the keys one by one, with P as it is in
            # fp32 where the product takes it in 16 bits: half a step of P times |v|, and the sums' own 2^-20.
            # Each result is rounded once.
            least = 0.0 if have >= 1000 else (2.0**-8 if fmt == "bf16" else 2.0**-11) + 2.0**-20 + 2 * UNIT[dtype]
            assert off.max() <= least * _largest_value(c, where)
        else:
            assert out[:, G:].isnan().all() and lse[:, G:].isnan().all()
        t[page, slot, 1] = old


@pytest.mark.parametrize("fmt,dtype", [f for f in FORMATS if f[0] != "e4m3"])
@pytest.mark.parametrize("T,G", [(3, 4), (40, 4)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
def test_an_infinite_value_of_little_weight_among_new_tokens(bad, T, G, fmt, dtype):
    """New token 0's score lies 300 powers of two below the others': its infinite value comes out of the
    rows that see it, and of no others."""
    c, q = _setup(T, G, 5, fmt, dtype)
    q.fill_(1.0)
    where = _slots(c, 0, 5 + T)
    c.k[where] = torch.full((), 4.0, device="cuda").to(c.k.dtype)
    c.k[where[0][5], where[1][5]] = torch.zeros((), device="cuda").to(c.k.dtype)
    mask = torch.full((T, 1), -1, dtype=torch.int64, device="cuda")
    mask[1] = -2   # (token 1 does not see it)
    c.v[where[0][5], where[1][5], 1, 3] = bad
    out = qlin.qlin_cache_attention(c, q, 300 / (4 * D) * math.log(2), mask)
    assert qlin.qlin_sync_status() == 0
    sees = torch.arange(T, device="cuda") != 1
    assert (out[sees][:, G:, 3] == bad).all()
    out[:, G:, 3][sees] = 0.0
    assert out.isfinite().all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,G,have", FORMS)
def test_key_scales_of_any_sign(T, G, have, dtype):
    c, q = _setup(T, G, have, "e4m3", dtype)
    c.k_scale.neg_()
    out, lse = _call(c, q)
    _check(c, q, 0.125, None, "e4m3", out, lse)
    # the same values from codes of the other sign
    other = qlin.PagedCache(**(vars(c) | dict(k=(c.k.view(torch.uint8) ^ 0x80).view(c.k.dtype), k_scale=-c.k_scale)))
    same, same_lse = _call(other, q)
    assert torch.equal(out, same) and torch.equal(lse, same_lse)
    for zero in (0.0, -0.0):
        c.k_scale.fill_(zero)
        out, lse = _call(c, q)
        _check(c, q, 0.125, None, "e4m3", out, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,G,have", FORMS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_scales_that_are_not_finite_give_nan(bad, T, G, have, dtype):
    c, q = _setup(T, G, have, "e4m3", dtype)
    c.k_scale.fill_(bad)
    out, lse = _call(c, q)
    assert out.isnan().all() and lse.isnan().all()


def test_rows_that_see_nothing_whatever_the_scale_and_the_query():
    for T, G in ((1, 4), (40, 4)):
        c, q = _setup(T, G, 0, "e4m3", torch.bfloat16)
        q[0, 0, 0] = math.nan
        for scale in (math.nan, math.inf, -1.0, 6 / 448):
            c.k_scale.fill_(scale)
            lse = torch.full(q.shape[:2], 5.0, device="cuda")
            out = qlin.qlin_cache_attention(c, q, 0.125, torch.zeros(T, 1, dtype=torch.int64, device="cuda"), lse=lse)
            assert (out == 0).all() and (lse == -math.inf).all()
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("fmt,dtype", [f for f in FORMATS if f[0] != "e4m3"])
@pytest.mark.parametrize("T,G,have", FORMS)
def test_scores_of_minus_infinity(T, G, have, fmt, dtype):
    """Beside finite scores they weigh nothing; a row that sees no others comes out as one that sees
    no key."""
    c, q = _setup(T, G, have, fmt, dtype)
    q[..., 0] = 1.0
    where = _slots(c, 0, have + T)
    c.k[where + (slice(None), 0)] = -math.inf
    out, lse = _call(c, q)
    assert (out == 0).all() and (lse == -math.inf).all()
    c.k[where[0][1:], where[1][1:], :, 0] = 0.0
    out, lse = _call(c, q)
    assert out.isfinite().all() and lse.isfinite().all()
