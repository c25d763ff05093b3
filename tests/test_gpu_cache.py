"""Appending to a paged cache and the attention over it against their formulas in 64 bits.

Append: as the rotary positions, 2^-21 (|a| + |b|) times the magnitude and one rounding to
the cache's type (E4M3: of value / scale, whose reciprocal rounds once more).

Attention, relative to sum p |v| / sum p: a score's fp32 sum runs in steps of at least 8
elements, each 2^-23 of ||q|| ||k|| scale, and its scaling keeps 2^-22 of it (E4M3: Q in fp16
after a power of two is off by 2^-11 of an element or 2^-24 of the row's largest, the latter
only where the type of Q has more bits than fp16 there); exp2 keeps 2^-21.  P is rounded to
the values' type (2^-8 bf16, 2^-11 fp16 or, below fp16's normals, 2^-25), the sums over keys
run in steps of 16 keys at 2^-23 each and are joined in fp32."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
LEAST = {torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}
NAMES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _make(cached, new, heads, D, page, fmt, seed=0, spare=3, junk=float("nan"), grow=0):
    """A cache whose pages lie in random order among others; what no token reaches is junk."""
    g = _gen(seed)
    per = [max(1, -(-(c + n + grow) // page)) for c, n in zip(cached, new)]
    pages, width = sum(per) + spare, max(per) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(cached), width), -7, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    fp8 = fmt == "e4m3"
    c = qlin.PagedCache(*(torch.full((pages, page, heads, D), junk, device="cuda").to(NAMES[fmt]) for _ in "kv"),
                        table, _ints(cached), _ints([0] + list(np.cumsum(new))),
                        torch.tensor([6 / 448], device="cuda") if fp8 else None,
                        torch.tensor([5 / 448], device="cuda") if fp8 else None)
    return c


def _slots(c, b, n):
    """(page, slot) of the first n tokens of sequence b."""
    i = torch.arange(n, device="cuda")
    page = c.k.shape[1]
    return c.page_table[b, i // page].long(), i % page


def _fill(c, cached, new, seed=1):
    """Values in every slot that the sequences' tokens take."""
    g = _gen(seed)
    for b, n in enumerate(np.add(cached, new)):
        if n == 0:
            continue
        where = _slots(c, b, int(n))
        for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
            x = torch.randn(int(n), t.shape[2], t.shape[3], generator=g, device="cuda")
            t[where] = (x if s is None else (x / s).clamp(-448, 448)).to(t.dtype)


def _pack(bits):
    """bool [tokens, new] -> int64 words."""
    T, n = bits.shape
    words = max(1, -(-n // 64))
    b = torch.nn.functional.pad(bits, (0, 64 * words - n)).view(T, words, 64).cpu().numpy()
    w = (b.astype(np.uint64) << np.arange(64, dtype=np.uint64)).sum(2, dtype=np.uint64)
    return torch.from_numpy(w.view(np.int64)).cuda()


def _expected(c, q, scale, bits, fmt):
    """(out, lse, tolerance of out, of lse) in 64 bits."""
    T, Hq, D = q.shape
    H = c.k.shape[2]
    G = Hq // H
    starts, cached = c.q_start.tolist(), c.cached.tolist()
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda"), torch.full((T, Hq), -math.inf,
                                                                                   dtype=torch.float64, device="cuda")
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u = 2.0**-8 if fmt == "bf16" else 2.0**-11
    for b, have in enumerate(cached):
        t0, t1 = starts[b], starts[b + 1]
        n, L = t1 - t0, have + t1 - t0
        if n == 0:
            continue
        where = _slots(c, b, L)
        k, v = c.k[where].double(), c.v[where].double()
        if fmt == "e4m3":
            k, v = k * c.k_scale.double(), v * c.v_scale.double()
        see = torch.ones(n, L, dtype=torch.bool, device="cuda")
        see[:, have:] = bits[t0:t1, :n] if bits is not None else torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for h in range(Hq):
            kh, vh, qh = k[:, h // G], v[:, h // G], q[t0:t1, h].double()
            s = (qh @ kh.nan_to_num(0, 0, 0).t()) * scale
            s = s.masked_fill(~see, -math.inf)
            m = s.amax(1, keepdim=True)
            p = torch.exp(s - torch.where(torch.isinf(m), 0, m))
            total = p.sum(1, keepdim=True)
            some = total > 0
            vz = torch.where(see.any(0)[:, None], vh, torch.zeros_like(vh)).nan_to_num(0, 0, 0)
            inv = torch.where(some, 1 / total, 0)
            out[t0:t1, h], lse[t0:t1, h] = (p @ vz) * inv, (m + torch.log(total))[:, 0]
            size = scale * qh.norm(dim=1, keepdim=True) * kh.nan_to_num(0, 0, 0).norm(dim=1).max()
            eps = 2.0**-23 * (D / 8 + 4) * size + 2.0**-21 + (2.0**-24 * math.sqrt(D) * size if fmt == "e4m3" else 0)
            if fmt == "e4m3" and q.dtype is torch.bfloat16:
                eps = eps + 2.0**-24 * math.sqrt(D) * size
            rel = u + 2 * eps + (L / 16 + 64) * 2.0**-23
            tol[t0:t1, h] = rel * (p @ vz.abs()) * inv + (2.0**-25 * vz.abs().sum(0) if fmt != "bf16" else 0) * inv
            ltol[t0:t1, h] = (eps[:, 0] + (L / 16 + 64) * 2.0**-23 + 2.0**-22 + 2.0**-22 * lse[t0:t1, h].abs()
                              ).nan_to_num(0, 0, 0)
    return out, lse, tol, ltol


def _check(c, q, scale, bits, fmt, out, lse, rows=slice(None)):
    want, wl, tol, ltol = _expected(c, q, scale, bits, fmt)
    u = UNIT[q.dtype]
    off = ((out.double() - want).abs() - (tol + u * (want.abs() + tol) + LEAST[q.dtype]))[rows]
    assert not out[rows].isnan().any()
    assert off.max() <= 0, (off.max().item(), torch.nonzero(off > 0)[:4].tolist(), (off > 0).sum().item())
    if lse is not None:
        empty = torch.isinf(wl[rows])
        assert (lse[rows][empty] == -math.inf).all() and (out[rows][empty] == 0).all()
        bad = ((lse.double() - wl).abs() > ltol)[rows] & ~empty
        assert not bad.any(), (lse[rows][bad][:4], wl[rows][bad][:4])


def _attend(cached, new, heads, G, D, page, fmt, dtype, tree=True, seed=0, scale=None, density=0.5):
    c = _make(cached, new, heads, D, page, fmt, seed)
    _fill(c, cached, new, seed + 1)
    T = sum(new)
    q = torch.randn(T, heads * G, D, generator=_gen(seed + 2), device="cuda").to(dtype)
    bits = None
    if tree:
        bits = torch.rand(T, max(new), generator=_gen(seed + 3), device="cuda") < density
        bits[T - 1] = False                      # this token sees none of the new ones
    scale = scale or 1 / math.sqrt(D)
    lse = torch.full((T, heads * G), 5.0, device="cuda")
    out = qlin.qlin_cache_attention(c, q, scale, None if bits is None else _pack(bits), lse=lse)
    assert qlin.qlin_sync_status() == 0
    _check(c, q, scale, bits, fmt, out, lse)
    return c, q, bits, out


FORMATS = [("bf16", torch.bfloat16), ("fp16", torch.float16), ("e4m3", torch.bfloat16), ("e4m3", torch.float16)]


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("D", [16, 48, 64, 80, 96, 128, 144, 192, 256])
def test_head_dims(D, fmt, dtype):
    # a single token, short runs, a new sequence without a cache
    _attend([70, 0, 33], [1, 1, 1], 2, 4, D, 16, fmt, dtype, tree=False)
    _attend([70, 0, 33], [3, 7, 30], 2, 3, D, 16, fmt, dtype)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("page", [1, 3, 8, 64, 256])
@pytest.mark.parametrize("cached,new", [([0], [1]), ([1], [1]), ([63], [1]), ([64], [2]), ([127, 128, 129], [1, 1, 1]),
                                        ([5, 0, 200, 0], [0, 4, 0, 1]), ([300, 17, 1000], [65, 1, 129])])
def test_lengths_and_pages(cached, new, page, fmt, dtype):
    _attend(cached, new, 2, 2, 64, page, fmt, dtype)
    _attend(cached, new, 2, 2, 64, page, fmt, dtype, tree=False)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("heads,G", [(1, 1), (3, 5), (7, 1), (2, 8), (1, 16), (1, 33)])
def test_groups(heads, G, fmt, dtype):
    _attend([150, 400], [1, 1], heads, G, 128, 32, fmt, dtype, tree=False)
    _attend([150, 400], [13, 4], heads, G, 128, 32, fmt, dtype)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_long_caches_and_uneven_batches(fmt, dtype):
    _attend([30001], [1], 1, 8, 128, 16, fmt, dtype, tree=False)
    _attend([20000, 1, 9000, 0, 300], [2, 1, 5, 3, 1], 2, 4, 96, 64, fmt, dtype)
    _attend([40] * 200, [1] * 200, 2, 2, 64, 16, fmt, dtype, tree=False)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_many_sequences(fmt, dtype):
    # more than a CTA has threads, some without new tokens; a CTA's run over many items
    _attend([37 * i % 1500 for i in range(300)], [int(i % 7 > 0) for i in range(300)], 1, 2, 64, 16, fmt, dtype, tree=False)
    _attend([53 * i % 900 for i in range(700)], [i % 4 * 11 for i in range(700)], 1, 1, 64, 32, fmt, dtype)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_many_rows(fmt, dtype):
    _attend([1500, 700], [64, 33], 2, 4, 128, 128, fmt, dtype)
    _attend([900], [128], 1, 8, 64, 8, fmt, dtype)
    _attend([5000, 250], [128, 17], 2, 5, 80, 32, fmt, dtype, tree=False)
    _attend([0, 0], [100, 28], 2, 3, 128, 64, fmt, dtype, tree=False)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("D", [16, 64, 80, 96, 128, 160, 192, 256])
@pytest.mark.parametrize("page", [8, 24, 64, 128, 256])
def test_many_rows_head_dims_and_pages(page, D, fmt, dtype):
    # one half of the rows and two, tiles that end in a page, sequences without a cache
    _attend([130, 0, 515], [40, 9, 25], 2, 4, D, page, fmt, dtype)
    _attend([128, 64, 383, 0], [64, 128, 1, 33], 1, 4, D, page, fmt, dtype, tree=False)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("cached", [0, 1, 63, 64, 91, 92, 127, 128, 129, 255, 256, 300, 2000, 40000])
def test_many_rows_lengths(cached, fmt, dtype):
    _attend([cached], [36], 1, 3, 64, 16, fmt, dtype)
    _attend([cached, 7 * cached // 8], [130, 70], 1, 2, 128, 64, fmt, dtype)
    _attend([cached, 7 * cached // 8], [130, 70], 1, 2, 192, 32, fmt, dtype)
    _attend([cached // 2] * 70, [37] * 70, 3, 1, 64, 32, fmt, dtype, tree=False)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_empty_rows(fmt, dtype):
    # no cache and masks of nothing
    for D, T, heads, G in ((64, 9, 2, 3), (128, 100, 1, 4)):
        c = _make([0], [T], heads, D, 16, fmt)
        _fill(c, [0], [T])
        bits = torch.zeros(T, T, dtype=torch.bool, device="cuda")
        bits[2, 1] = bits[4, 4] = bits[T - 1, 0] = True
        q = torch.randn(T, heads * G, D, generator=_gen(5), device="cuda").to(dtype)
        lse = torch.empty(T, heads * G, device="cuda")
        out = qlin.qlin_cache_attention(c, q, 0.1, _pack(bits), lse=lse)
        _check(c, q, 0.1, bits, fmt, out, lse)
        assert (out[0] == 0).all() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T,G", [(6, 2), (70, 4)])
def test_what_is_not_seen_does_not_reach_a_row(T, G, bad, fmt, dtype):
    heads, D, have = 2, 64, 50
    if fmt == "e4m3" and not math.isnan(bad):
        pytest.skip("E4M3 has no infinity")
    c = _make([have], [T], heads, D, 16, fmt)
    _fill(c, [have], [T])
    bits = torch.rand(T, T, generator=_gen(3), device="cuda") < 0.5
    bits[:, 3] = False
    bits[4, 3] = True                      # token 4 alone sees new token 3
    where = _slots(c, 0, have + T)
    c.k[where[0][have + 3], where[1][have + 3]] = bad
    c.v[where[0][have + 3], where[1][have + 3]] = bad
    q = torch.randn(T, heads * G, D, generator=_gen(5), device="cuda").to(dtype)
    lse = torch.empty(T, heads * G, device="cuda")
    out = qlin.qlin_cache_attention(c, q, 0.125, _pack(bits), lse=lse)
    rows = torch.arange(T, device="cuda") != 4
    _check(c, q, 0.125, bits, fmt, out, lse, rows)
    # only the values: the one that sees them takes them up, the others stay
    c.k[where[0][have + 3], where[1][have + 3]] = torch.zeros((), device="cuda").to(c.k.dtype)
    out = qlin.qlin_cache_attention(c, q, 0.125, _pack(bits), lse=lse)
    _check(c, q, 0.125, bits, fmt, out, lse, rows)
    assert out[4].isnan().all() if math.isnan(bad) else (out[4] == bad).all()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_scores_far_apart(fmt, dtype):
    # maxima that move from key to key, and large magnitudes
    for T, G in ((1, 4), (40, 4)):
        c = _make([700], [T], 1, 64, 32, fmt)
        _fill(c, [700], [T])
        where = _slots(c, 0, 700 + T)
        grow = torch.linspace(0.01, 3.0, 700 + T, device="cuda")[:, None, None]
        c.k[where] = (c.k[where].float() * grow).clamp(-448, 448).to(c.k.dtype)   # (E4M3: NaN above)
        q = (torch.randn(T, G, 64, generator=_gen(5), device="cuda") * 8).to(dtype)
        lse = torch.empty(T, G, device="cuda")
        out = qlin.qlin_cache_attention(c, q, 0.3, lse=lse)
        _check(c, q, 0.3, None, fmt, out, lse)


def test_bf16_queries_over_fp8_keys_at_any_magnitude():
    c = _make([200], [2], 1, 128, 16, "e4m3")
    _fill(c, [200], [2])
    for size in (1e-30, 1e-6, 1.0, 1e5, 1e30):
        q = (torch.randn(2, 4, 128, generator=_gen(5), device="cuda") * size).to(torch.bfloat16)
        lse = torch.empty(2, 4, device="cuda")
        out = qlin.qlin_cache_attention(c, q, 0.1 / size, lse=lse)
        _check(c, q, float(np.float32(0.1 / size)), None, "e4m3", out, lse)


@pytest.mark.parametrize("T,G", [(1, 4), (40, 4)])
def test_strides_and_padding(T, G):
    # q and out inside wider tensors, heads outermost in the cache, tokens behind the last
    # sequence, and an output over q
    heads, D = 2, 64
    cached, new = [100, 30], [T, T]
    c = _make(cached, new, heads, D, 16, "bf16")
    _fill(c, cached, new)
    n = 2 * T
    big = torch.randn(n + 3, heads * G + 2 * heads, D, generator=_gen(1), device="cuda").to(torch.bfloat16)
    q = big[:, :heads * G]
    plain = qlin.qlin_cache_attention(c, q[:n].contiguous(), 0.125)
    _check(c, q[:n], 0.125, None, "bf16", plain, None)
    wide = torch.full((n + 3, heads * G + 1, D + 16), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n + 3, heads * G), 9.0, device="cuda")
    qlin.qlin_cache_attention(c, q, 0.125, out=wide[:, 1:, :D], lse=lse)
    assert torch.equal(wide[:n, 1:, :D], plain)
    assert (wide[n:] == 9).all() and (wide[:, 0] == 9).all() and (wide[..., D:] == 9).all() and (lse[n:] == 9).all()
    other = qlin.PagedCache(c.k.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3),
                            c.v.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3), c.page_table, c.cached, c.q_start)
    assert torch.equal(qlin.qlin_cache_attention(other, q, 0.125)[:n], plain)
    mine = q[:n].contiguous()
    qlin.qlin_cache_attention(c, mine, 0.125, out=mine)
    assert torch.equal(mine, plain)
    assert qlin.qlin_sync_status() == 0


def test_bad_tables_and_counts_are_reported_and_touch_nothing():
    heads, D = 2, 64
    for T, G in ((1, 4), (40, 4)):
        c = _make([100, 30], [T, T], heads, D, 16, "bf16")
        _fill(c, [100, 30], [T, T])
        q = torch.randn(2 * T, heads * G, D, generator=_gen(1), device="cuda").to(torch.bfloat16)
        good = qlin.qlin_cache_attention(c, q, 0.125)
        kv = torch.randn(2 * T, heads, D, generator=_gen(2), device="cuda").to(torch.bfloat16)
        for page in (-1, c.k.shape[0], 2**31 - 1, -2**31):
            t = c.page_table.clone()
            t[0, 6] = page                       # keys 96 .. 111 of the first sequence
            bad = qlin.PagedCache(c.k.clone(), c.v.clone(), t, c.cached, c.q_start)
            out = qlin.qlin_cache_attention(bad, q, 0.125)
            assert qlin.qlin_sync_status() == 1
            assert torch.equal(out[T:], good[T:]) and not out.isnan().any()
            qlin.qlin_cache_append(bad, kv, kv)
            assert qlin.qlin_sync_status() == 1
            where = _slots(c, 1, 30 + T)
            assert torch.equal(bad.k[where[0][30:], where[1][30:]], kv[T:])
        for cached, start in (([-1, 30], [0, T, 2 * T]), ([10**6, 30], [0, T, 2 * T]), ([100, 30], [T, 0, 2 * T]),
                              ([100, 30], [0, T, 2 * T + 5]), ([2**31 - 1, 30], [0, T, 2 * T])):
            bad = qlin.PagedCache(c.k.clone(), c.v.clone(), c.page_table, _ints(cached), _ints(start))
            qlin.qlin_cache_attention(bad, q, 0.125)
            assert qlin.qlin_sync_status() == 1
            qlin.qlin_cache_append(bad, kv, kv)
            assert qlin.qlin_sync_status() == 1
        ws = qlin.alloc_cache_attention_workspace()
        assert torch.equal(qlin.qlin_cache_attention(c, q, 0.125, workspace=ws), good)
        assert qlin.qlin_sync_status() == 0 and (ws[:8192] == 0).all()


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("D,G,parts", [(64, 1, 64), (64, 16, 32), (256, 16, 16)])
def test_items_that_meet_in_a_cta(D, G, parts, fmt, dtype):
    """One sequence's last CTA begins the next one, and is alone in its group of `parts` CTAs
    that join their sums.  (Two tiles each, for the tiles and grids that there may be.)"""
    ws = qlin.alloc_cache_attention_workspace()
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for tile in (32, 64, 128):
        for ctas in (sms, 2 * sms):
            n = 2 * parts + 1
            cached = [n * tile - 1, (2 * ctas - n) * tile - 1]
            c = _make(cached, [1, 1], 1, D, 64, fmt, tile)
            _fill(c, cached, [1, 1], tile + 1)
            q = torch.randn(2, G, D, generator=_gen(tile + 2), device="cuda").to(dtype)
            first = qlin.qlin_cache_attention(c, q, 1 / math.sqrt(D), workspace=ws)
            assert not ws[:8192].any()
            _check(c, q, 1 / math.sqrt(D), None, fmt, first, None)
            for _ in range(5):
                assert torch.equal(qlin.qlin_cache_attention(c, q, 1 / math.sqrt(D), workspace=ws), first)
            assert not ws[:8192].any()


@pytest.mark.parametrize("T,G", [(1, 4), (40, 4)])
def test_graph_over_growing_sequences_and_streams(T, G):
    heads, D, B = 2, 128, 3
    cached, new = [100, 500, 3], [T, T, T]
    c = _make(cached, new, heads, D, 16, "bf16", grow=600)
    _fill(c, [n + 600 for n in cached], new)
    q = torch.randn(B * T, heads * G, D, generator=_gen(1), device="cuda").to(torch.bfloat16)
    ws, out = qlin.alloc_cache_attention_workspace(), torch.empty_like(q)
    qlin.qlin_cache_attention(c, q, 0.1, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qlin.qlin_cache_attention(c, q, 0.1, out=out, workspace=ws)
        qlin.qlin_cache_attention(c, q, 0.1, out=out, workspace=ws)
    s = torch.cuda.Stream()
    for grow in (0, 1, 37, 600):
        c.cached.copy_(_ints([n + grow for n in cached]))
        graph.replay()
        torch.cuda.synchronize()
        _check(c, q, 0.1, None, "bf16", out, None)
        eager = qlin.qlin_cache_attention(c, q, 0.1, stream=s)
        s.synchronize()
        assert torch.equal(eager, out)
        # two at once, each with its workspace
        one = qlin.qlin_cache_attention(c, q, 0.1, workspace=ws)
        two = qlin.qlin_cache_attention(c, q, 0.1, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(one, out) and torch.equal(two, out)
    assert qlin.qlin_sync_status() == 0


def test_offsets_past_32_bits():
    # pages beyond 2^32 bytes of a cache
    heads, D, page = 8, 128, 256
    pages = (5 << 30) // (page * heads * D * 2)
    c = _make([1], [1], heads, D, page, "bf16")
    k = torch.zeros(pages, page, heads, D, dtype=torch.bfloat16, device="cuda")
    far = qlin.PagedCache(k, k, _ints([[pages - 1, pages - 2, 0]]), _ints([300]), _ints([0, 2]))
    new = torch.randn(2, heads, D, generator=_gen(1), device="cuda").to(torch.bfloat16)
    qlin.qlin_cache_append(far, new, new)
    assert torch.equal(k[pages - 2, 44:46], new) and (k[:pages - 2] == 0).all()
    q = torch.randn(2, heads, D, generator=_gen(2), device="cuda").to(torch.bfloat16)
    _check(far, q, 0.1, None, "bf16", qlin.qlin_cache_attention(far, q, 0.1), None)
    del c


# ------------------------------------------------------------------ append ---

def _turned(x, pos, plan):
    """(rotated in 64 bits, |a| + |b| of each element's pair)."""
    T, H, D = x.shape
    R, half = plan.rot_dim, plan.rot_dim // 2
    turns = [int(v) for v in plan.turns.cpu().numpy().view(np.uint64)]
    axis = np.repeat(np.arange(len(plan.axis_pairs)), plan.axis_pairs)
    pos = pos.cpu().numpy().reshape(T, -1)
    frac = np.array([[((int(pos[t, axis[i]]) * turns[i]) % 2**64) / 2**64 for i in range(half)] for t in range(T)])
    ang = torch.from_numpy(frac * 2 * math.pi).to(x.device)[:, None]
    co, si, m = torch.cos(ang), torch.sin(ang), plan.magnitude
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    i = torch.arange(half, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if plan.layout == "interleaved" else (i, i + half)
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = m * (a * co - b * si), m * (a * si + b * co)
    size[..., ia] = size[..., ib] = m * (a.abs() + b.abs())
    return y, size


def _near(got, want, size, scale=None):
    if got.dtype is torch.float8_e4m3fn:
        s = scale.double()
        w, e = want / s, (2.0**-21 * size + 2.0**-22 * want.abs()) / s
        lo, hi = (w - e).clamp(-448, 448), (w + e).clamp(-448, 448)
        # the code of a value between lo and hi (by their own roundings: 2^-4 or 2^-10 apart at most)
        off = (got.double() - w.clamp(-448, 448)).abs() - (2.0**-4 * torch.maximum(lo.abs(), hi.abs()) + e + 2.0**-10)
    else:
        off = (got.double() - want).abs() - (UNIT[got.dtype] * want.abs() + (1 + UNIT[got.dtype]) * 2.0**-21 * size
                                            + LEAST[got.dtype])
    assert off.max() <= 0, off.max().item()


def _append(cached, new, heads, Hq, D, page, fmt, dtype, plan, pos, packed=True, seed=0, pad=2, shift=0):
    c = _make(cached, new, heads, D, page, fmt, seed, junk=1.5)
    T = sum(new) + pad
    base = torch.randn(T, (Hq + 2 * heads) * D + shift, generator=_gen(seed), device="cuda").to(dtype)
    qkv = base[:, shift:].view(T, Hq + 2 * heads, D)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:]
    if not packed:
        q, k, v = (t.contiguous() for t in (q, k, v))
    before = c.k.clone(), c.v.clone()
    q_out = torch.full((T, Hq, D), 7.0, dtype=dtype, device="cuda") if Hq else None
    qlin.qlin_cache_append(c, k, v, plan, pos, q if Hq else None, q_out)
    assert qlin.qlin_sync_status() == 0
    n = sum(new)
    at = torch.cat([torch.arange(a, a + b) for a, b in zip(cached, new)]).cuda()
    p = pos[:n] if pos is not None else at
    if plan is None:
        kr, ks, qr, qs = k[:n].double(), 0 * k[:n].double(), q[:n].double(), 0 * q[:n].double()
    else:
        (kr, ks), (qr, qs) = _turned(k[:n], p, plan), _turned(q[:n], p, plan) if Hq else (None, None)
    places = [torch.cat(t) for t in zip(*[[x[a:a + b] for x in _slots(c, i, a + b)]
                                          for i, (a, b) in enumerate(zip(cached, new)) if b])]
    _near(c.k[places[0], places[1]], kr, ks, c.k_scale)
    _near(c.v[places[0], places[1]], v[:n].double(), 0 * v[:n].double(), c.v_scale)
    if Hq:
        _near(q_out[:n], qr, qs)
        assert (q_out[n:] == 7).all()
    # every other slot as it was
    for t, old in ((c.k, before[0]), (c.v, before[1])):
        t[places[0], places[1]] = old[places[0], places[1]]
        assert torch.equal(t.view(torch.uint8), old.view(torch.uint8))


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,Hq,D,R", [(2, 4, 64, 64), (1, 1, 128, 64), (3, 0, 128, 128), (8, 24, 128, 128), (2, 6, 80, 40),
                                          (1, 7, 256, 256), (2, 4, 96, 48), (1, 3, 66, 34), (5, 5, 2, 2), (2, 2, 48, 20)])
def test_append(heads, Hq, D, R, layout, fmt, dtype):
    plan = qlin.rope_plan(R, layout=layout)
    pos = torch.randint(0, 1 << 17, (40,), generator=_gen(2), device="cuda")
    _append([0, 17, 5, 3], [3, 1, 0, 34], heads, Hq, D, 8, fmt, dtype, plan, pos)
    _append([0, 17, 5, 3], [3, 1, 0, 34], heads, Hq, D, 5, fmt, dtype, plan, None, packed=False, shift=1)
    _append([250], [1], heads, Hq, D, 64, fmt, dtype, None if Hq else plan, None, packed=True, pad=0)


@pytest.mark.parametrize("fmt,dtype", FORMATS)
def test_append_axes_scalings_and_batches(fmt, dtype):
    plan = qlin.rope_plan((16, 56, 56), layout="interleaved", scaling="yarn", factor=8.0)
    pos = torch.randint(-50, 1 << 17, (702, 3), generator=_gen(2), device="cuda").to(torch.int32)
    _append([0], [700], 24, 24, 128, 64, fmt, dtype, plan, pos)
    _append([7 * b for b in range(200)], [1 + b % 3 for b in range(200)], 2, 4, 64, 16, fmt, dtype,
            qlin.rope_plan(64, scaling="ntk", factor=4.0), None)


def test_append_in_place_and_in_a_graph():
    heads, Hq, D, B = 2, 4, 128, 5
    c = _make([10, 0, 3, 60, 7], [1] * B, heads, D, 16, "bf16", junk=0.0, grow=8)
    plan = qlin.rope_plan(D)
    qkv = torch.randn(B, Hq + 2 * heads, D, generator=_gen(1), device="cuda").to(torch.bfloat16)
    src = qkv.clone()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:]
    want = qlin.qlin_cache_append(c, k, v, plan, None, q)
    qlin.qlin_cache_append(c, k, v, plan, None, q, q)
    assert torch.equal(q, want) and torch.equal(k, src[:, Hq:Hq + heads])
    # k as the rotary call turns it at the same positions
    at = c.cached.long()
    turned = qlin.qlin_rope(k, at, plan)
    for b in range(B):
        w = _slots(c, b, int(at[b]) + 1)
        assert torch.equal(c.k[w[0][-1], w[1][-1]], turned[b])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    q_out = torch.empty_like(want)
    with torch.cuda.graph(graph):
        qlin.qlin_cache_append(c, k, v, plan, None, src[:, :Hq], q_out)
        c.cached.add_(1)
    for _ in range(3):
        at = c.cached.long()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, qlin.qlin_rope(src[:, :Hq], at, plan))
        turned = qlin.qlin_rope(k, at, plan)
        for b in range(B):
            w = _slots(c, b, int(at[b]) + 1)
            assert torch.equal(c.k[w[0][-1], w[1][-1]], turned[b]) and torch.equal(c.v[w[0][-1], w[1][-1]], v[b])


# --------------------------------------------------------- a step of them ---

@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_a_serving_step(fmt):
    """Quantizer, QKV, append, attention of a draft and the out-projection in a row, captured
    once and replayed as the sequences grow, against the same step of single calls' formulas."""
    heads, G, D, page, hidden = 2, 4, 64, 16, 512
    cached, T = [200, 31, 0], 5
    B, n = len(cached), len(cached) * T
    c = _make(cached, [T] * B, heads, D, page, fmt, grow=64)
    _fill(c, [x + 64 for x in cached], [T] * B)
    g = _gen(3)
    weight = lambda o, i: qlin.qlin_quantize_fp8_block(  # noqa: E731
        (torch.randn(o, i, generator=g, device="cuda") / math.sqrt(i)).to(torch.bfloat16), 128)
    wqkv, wout = weight((G + 2) * heads * D, hidden), weight(hidden, G * heads * D)
    plan, ws = qlin.rope_plan(D, scaling="yarn", factor=4.0), qlin.alloc_cache_attention_workspace()
    bits = torch.ones(n, T, dtype=torch.bool, device="cuda").view(B, T, T).tril().view(n, T)
    bits[::T, 1:] = False
    bits[3::T, 2] = False
    mask = _pack(bits)
    x = torch.randn(n, hidden, generator=g, device="cuda").to(torch.bfloat16)
    captured, eager = {}, {}

    def step(state):
        a = qlin.qlin_quantize_fp8_block(x)
        qkv = qlin.qlin_linear_fp8_block(a, wqkv).view(n, (G + 2) * heads, D)
        q = qlin.qlin_cache_append(c, qkv[:, G * heads:(G + 1) * heads], qkv[:, (G + 1) * heads:], plan, None,
                                   qkv[:, :G * heads])
        o = qlin.qlin_cache_attention(c, q, 1 / math.sqrt(D), mask, workspace=ws)
        y = qlin.qlin_linear_fp8_block(qlin.qlin_quantize_fp8_block(o.view(n, -1)), wout, residual=x)
        state.update(q=q, o=o, y=y, qkv=qkv)

    step(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(captured)
    for grow in (0, 3, 64):
        c.cached.copy_(_ints([v + grow for v in cached]))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in captured.items()}
        _check(c, got["q"], 1 / math.sqrt(D), bits, fmt, got["o"], None)
        at = torch.cat([torch.arange(v + grow, v + grow + T) for v in cached]).cuda()
        assert torch.equal(got["q"], qlin.qlin_rope(got["qkv"][:, :G * heads].contiguous(), at, plan))
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got["y"], eager["y"]) and torch.isfinite(got["y"].float()).all()
    assert qlin.qlin_sync_status() == 0
