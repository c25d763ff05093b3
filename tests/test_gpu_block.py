"""The transformer block: its forward against the calls made one by one, a captured
graph, and the unquantized block in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import block, qlin

pytestmark = pytest.mark.gpu

H, HEADS, F = 512, 8, 1088


def _make(fmt, M, seed=3):
    b = block.build_block(fmt, M, H, HEADS, F, axes=(16, 24, 24), seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(M, H, generator=g, device="cuda").bfloat16()
    pos = torch.randint(0, 64, (M, 3), generator=g, device="cuda", dtype=torch.int32)
    b.calibrate(x)
    return b, x, pos


@pytest.mark.parametrize("fmt", ["fp8", "nvfp4"])
@pytest.mark.parametrize("M", [1, 9, 77, 700])
def test_forward_is_its_calls(fmt, M):
    b, x, pos = _make(fmt, M)
    y = b.forward(x, pos).clone()
    assert qlin.qlin_sync_status() == 0 and torch.isfinite(y.float()).all()
    lin = qlin.qlin_linear_fp8 if fmt == "fp8" else qlin.qlin_linear_nvfp4
    def norm(v, w, name, r=None):
        if fmt == "fp8":
            return qlin.qlin_rmsnorm_fp8(v, w, r, block.EPS)
        return qlin.qlin_rmsnorm_nvfp4(v, b.scale[name], w, r, block.EPS)
    alloc = (lambda k: qlin.alloc_fp8(M, k, False)) if fmt == "fp8" else (lambda k: qlin.alloc_nvfp4(M, k))
    a, _ = norm(x, b.norm1, "a")
    vq, uq = alloc(H), alloc(F)
    qkv = torch.empty(M, 3 * H, dtype=torch.bfloat16, device="cuda")
    lin(a, b.W["qkv"], b.bias["qkv"], y=qkv, next_scale=b.scale["v"], y_q=vq, rq_col0=2 * H)
    rot = qlin.qlin_rope(qkv.view(M, 3 * HEADS, H // HEADS)[:, :2 * HEADS], pos, b.plan)
    assert torch.equal(b.qkv.view(M, 3 * HEADS, -1)[:, :2 * HEADS], rot)
    assert torch.equal(b.qkv[:, 2 * H:], qkv[:, 2 * H:])
    o, _ = lin(vq, b.W["out"], b.bias["out"])
    c, x1 = norm(o, b.norm2, "c", x)
    lin(c, b.W["up"], b.bias["up"], qlin.QLIN_ACT_GELU_TANH, next_scale=b.scale["u"], y_q=uq)
    y2, _ = lin(uq, b.W["down"], b.bias["down"], residual=x1)
    assert torch.equal(y, y2) and torch.equal(b.x1, x1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.forward(x, pos)
    b.y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b.y, y)


# Rounding errors of the two formats per operand, as shares of its norm: E4M3 2^-4 / sqrt
# 12 times a spread of at most 2 inside a binade and scales that leave small values
# subnormal, 4%; e2m1 with block scales 12%.  Two operands each in three linears on the
# way to y - x, added as if all errors aligned.
@pytest.mark.parametrize("fmt,per_operand", [("fp8", 0.04), ("nvfp4", 0.12)])
def test_against_the_unquantized_block(fmt, per_operand):
    M = 77
    g = torch.Generator(device="cuda").manual_seed(11)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = {"qkv": rnd(3 * H, H) / math.sqrt(H), "out": rnd(H, H) / math.sqrt(H), "up": rnd(F, H) / math.sqrt(H),
         "down": rnd(H, F) / math.sqrt(F), "norm1": 1 + 0.1 * rnd(H), "norm2": 1 + 0.1 * rnd(H)}
    w |= {n + ".bias": 0.1 * rnd(w[n].shape[0]) for n in ("qkv", "out", "up", "down")}
    w = {n: v.bfloat16() for n, v in w.items()}
    b = block.build_block(fmt, M, H, HEADS, F, weights=w)
    x = rnd(M, H).bfloat16()
    pos = torch.arange(M, device="cuda", dtype=torch.int32)
    b.calibrate(x)
    y = b.forward(x, pos).double()
    d = {n: v.double() for n, v in w.items()}
    rms = lambda v, n: v / torch.sqrt(v.square().mean(1, keepdim=True) + block.EPS) * d[n]  # noqa: E731
    lin = lambda v, n: v @ d[n].t() + d[n + ".bias"]  # noqa: E731
    xd = x.double()
    values = lin(rms(xd, "norm1"), "qkv")[:, 2 * H:]
    x1 = xd + lin(values, "out")
    u = lin(rms(x1, "norm2"), "up")
    u = u * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (u + 0.044715 * u**3))
    want = x1 + lin(u, "down")
    off = ((y - want).norm() / (want - xd).norm()).item()
    assert off <= 6 * per_operand, off
    # with attention's output given, here the values: the same block, the out-projection's
    # input quantized by its own scale
    q, k, v = b.project(x, pos)
    y2 = b.finish(x, v.reshape(M, H).contiguous()).double()
    assert ((y2 - want).norm() / (want - xd).norm()).item() <= 6 * per_operand
    assert q.shape == k.shape == v.shape == (M, HEADS, H // HEADS)


def test_refusals():
    with pytest.raises(ValueError):
        block.build_block("int8", 4, H, HEADS, F)
    with pytest.raises(ValueError):
        block.build_block("fp8", 4, H, 7, F)


def _paged(counts, cached, dtype, page=16):
    """A cache for sequences of `cached` tokens and `counts` new ones, pages back to front."""
    D = H // HEADS
    per = [-(-(c + n) // page) for c, n in zip(cached, counts)]
    table = torch.zeros(len(per), max(per), dtype=torch.int32, device="cuda")
    at = sum(per)
    for b, n in enumerate(per):
        table[b, :n] = torch.arange(at - 1, at - 1 - n, -1)
        at -= n
    g = torch.Generator(device="cuda").manual_seed(5)
    kv = [torch.randn(sum(per), page, HEADS, D, generator=g, device="cuda").to(dtype) for _ in "kv"]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    scale = torch.full((1,), 4 / 448, device="cuda") if dtype is torch.float8_e4m3fn else None
    starts = [sum(counts[:i]) for i in range(len(counts) + 1)]
    return qlin.PagedCache(*kv, table, ints(cached), ints(starts), scale, scale)


@pytest.mark.parametrize("fmt,dtype", [("fp8", torch.bfloat16), ("nvfp4", torch.float8_e4m3fn)])
@pytest.mark.parametrize("counts,cached,M", [([1], [40], 1), ([1, 1, 1], [0, 130, 15], 4), ([70, 0, 25], [33, 5, 0], 100)])
def test_step_is_its_calls(fmt, dtype, counts, cached, M):
    b, x, pos = _make(fmt, M)
    cache, again = (_paged(counts, cached, dtype) for _ in "ab")
    n = sum(counts)
    y = b.step(x, pos, cache).clone()
    attended = b.attended.clone()
    assert qlin.qlin_sync_status() == 0 and torch.isfinite(y.float()).all()
    q, k, v = b.project(x, pos)
    qlin.qlin_cache_append(again, k, v)
    o = qlin.qlin_cache_attention(again, q, (H // HEADS) ** -0.5)
    assert torch.equal(cache.k.view(torch.uint8), again.k.view(torch.uint8))
    assert torch.equal(cache.v.view(torch.uint8), again.v.view(torch.uint8))
    assert torch.equal(attended[:n], o.view(M, H)[:n]) and not attended[n:].any()
    assert torch.equal(b.finish(x, attended), y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(x, pos, cache)
    b.y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(b.y, y)


def test_attend_is_not_captured_first():
    b, x, pos = _make("fp8", 1)
    cache = _paged([1], [40], torch.bfloat16)
    q, k, v = b.project(x, pos)
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="captured"):
            b.attend(cache, q, k, v)
        b.y.zero_()
