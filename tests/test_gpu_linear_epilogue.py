"""The linears with bias, activation and residual against the formula in 64 bits.

Tolerances, before the rounding to 16 bits.  A product sum runs in fp32 steps of at
least 16 elements; each step rounds or truncates the running sum, which never exceeds
||a|| ||w||, by 2^-23 of it at most: (K / 16 + 8) 2^-23 ||a|| ||w||.  The activations'
slope is at most 1.13; exponentials, quotients and the three additions keep 2^-18 of
the values they meet."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle
from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from gpu_util import assert_requant_exact, bf16_bits, nvfp4_to_host, u8

FORMATS = ["nvfp4", "fp8", "fp8_rows", "bf16", "fp16"]
ACTS = [qlin.QLIN_ACT_NONE, qlin.QLIN_ACT_RELU, qlin.QLIN_ACT_SILU, qlin.QLIN_ACT_GELU_TANH, qlin.QLIN_ACT_GELU]
E2M1 = [0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6]


def _act(v, act):
    if act == qlin.QLIN_ACT_RELU:
        return v.clamp(min=0)
    if act == qlin.QLIN_ACT_SILU:
        return v * torch.sigmoid(v)
    if act == qlin.QLIN_ACT_GELU_TANH:
        return v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v**3))
    if act == qlin.QLIN_ACT_GELU:
        return v * 0.5 * torch.erfc(-v / math.sqrt(2))
    return v


def _values(q):
    """An operand's values in 64 bits."""
    if isinstance(q, torch.Tensor):
        return q.double()
    if isinstance(q, qlin.FP8Tensor):
        return q.codes.view(torch.float8_e4m3fn).double() * q.scale.double().view(-1, 1)
    canon = oracle.unswizzle_scales(u8(q.scales), q.rows, q.K)
    s = torch.from_numpy(np.ascontiguousarray(canon)).cuda().view(torch.float8_e4m3fn).double() * q.tensor_scale.double()
    grid = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    c = torch.stack([grid[(q.codes & 15).long()], grid[(q.codes >> 4).long()]], 2)
    return (c.view(q.rows, -1, 16) * s[..., None]).view(q.rows, q.K)


def _operands(fmt, M, N, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    a, w = rnd(M, K) * torch.exp(0.5 * rnd(M, 1)), rnd(N, K) / math.sqrt(K)
    dt = torch.float16 if fmt == "fp16" else torch.bfloat16
    a, w = a.to(dt), w.to(dt)
    if fmt == "nvfp4":
        a, w = qlin.qlin_quantize_act_nvfp4(a), qlin.qlin_quantize_weight(w, qlin.QLIN_FMT_NVFP4)
    elif fmt == "fp8":
        a, w = qlin.qlin_quantize_act_fp8(a), qlin.qlin_quantize_weight(w, qlin.QLIN_FMT_FP8)
    elif fmt == "fp8_rows":   # the weights' quantizer gives one scale per row
        a, w = qlin.qlin_quantize_weight(a, qlin.QLIN_FMT_FP8), qlin.qlin_quantize_weight(w, qlin.QLIN_FMT_FP8)
    return a, w, rnd(N).to(dt), rnd(M, N).to(dt), dt


def _call(fmt, *args, **kw):
    name = {"nvfp4": "qlin_linear_nvfp4", "bf16": "qlin_linear_bf16", "fp16": "qlin_linear_fp16"}.get(fmt, "qlin_linear_fp8")
    r = getattr(qlin, name)(*args, **kw)
    return r[0] if isinstance(r, tuple) else r


def _check(y, a, w, bias, act, residual, what):
    A, W = _values(a), _values(w)
    v = A @ W.t()
    K = A.shape[1]
    tol = (K / 16 + 8) * 2.0**-23 * 1.13 * A.norm(dim=1)[:, None] * W.norm(dim=1)
    if bias is not None:
        v = v + bias.double()
    tol = tol + 2.0**-18 * v.abs()
    v = _act(v, act)
    if residual is not None:
        v = v + residual.double()
        tol = tol + 2.0**-18 * residual.double().abs()
    u, low = (2.0**-11, 2.0**-25) if y.dtype == torch.float16 else (2.0**-8, 2.0**-134)
    off = (y.double() - v).abs() - (u * v.abs() + (1 + u) * tol + low)
    assert off.max() <= 0, (what, off.max().item(), tuple(x.item() for x in torch.where(off == off.max())))


# one token and a few; partial tiles; long and short K; each tile configuration
SHAPES = [(1, 64, 64), (1, 1024, 2560), (2, 192, 3136), (5, 576, 1088), (8, 3072, 512), (9, 64, 12288), (16, 320, 192),
          (17, 2112, 320), (33, 1024, 4160), (77, 320, 192), (129, 576, 1088), (300, 128, 512), (1300, 3648, 320),
          (2048, 4096, 1088), (552, 64, 4160), (1000, 576, 1088), (1040, 128, 320), (1500, 64, 1088),
          (300, 1024, 4160), (352, 320, 12288), (555, 832, 6208), (300, 3136, 6080),
          (1333, 2112, 320), (900, 2560, 1088)]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_shapes(M, N, K, fmt):
    a, w, bias, res, dt = _operands(fmt, M, N, K, M + N + K)
    act = ACTS[(M + N // 64 + K // 64) % 5]
    y = _call(fmt, a, w, bias, act, res)
    assert qlin.qlin_sync_status() == 0
    _check(y, a, w, bias, act, res, (fmt, M, N, K, act))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [1, 6, 200, 1000, 1333, 2048])
def test_parts(M, fmt):
    N, K = (4096, 192) if M == 2048 else (2112, 192) if M == 1333 else (448, 1088)
    a, w, bias, res, dt = _operands(fmt, M, N, K, 17 + M)
    for act in ACTS:
        for b, r in ((bias, None), (None, res), (None, None)):
            _check(_call(fmt, a, w, b, act, r), a, w, b, act, r, (fmt, M, act, b is None, r is None))


@pytest.mark.parametrize("fmt", ["nvfp4", "fp8", "bf16", "fp16"])
@pytest.mark.parametrize("M", [900, 2048])
def test_without_an_epilogue_as_the_plain_gemm(M, fmt):
    # at these sizes the same kernel runs: bit for bit
    N, K = (4096, 1088) if M == 2048 else (320, 960)
    a, w, _, _, _ = _operands(fmt, M, N, K, 3)
    plain = getattr(qlin, "qlin_gemm_" + fmt)(a, w)
    assert torch.equal(_call(fmt, a, w), plain)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M", [1, 7, 100, 1000, 1333, 2048])
def test_residual_in_place_and_strided(M, fmt):
    N, K = 4096 if M == 2048 else 2112 if M == 1333 else 320, 512
    a, w, bias, res, dt = _operands(fmt, M, N, K, 23)
    y0 = _call(fmt, a, w, bias, qlin.QLIN_ACT_SILU, res)
    y1 = res.clone()
    _call(fmt, a, w, bias, qlin.QLIN_ACT_SILU, y1, y1)
    assert torch.equal(y0, y1)
    wide = torch.zeros(M, N + 24, dtype=dt, device="cuda")
    wide[:, 8:8 + N] = res
    assert torch.equal(_call(fmt, a, w, bias, qlin.QLIN_ACT_SILU, wide[:, 8:8 + N]), y0)
    # an output that is only 16-byte aligned, nothing written beside it
    flat = torch.full((M * N + 16,), 5.0, dtype=dt, device="cuda")
    _call(fmt, a, w, bias, qlin.QLIN_ACT_SILU, res, flat[8:8 + M * N].view(M, N))
    assert torch.equal(flat[8:8 + M * N].view(M, N), y0) and (flat[:8] == 5).all() and (flat[-8:] == 5).all()


@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (3, 320, 1088), (16, 1024, 512), (40, 576, 320), (333, 512, 1088),
                                   (2048, 4096, 320), (700, 64, 2112),
                                   (352, 640, 12288), (555, 832, 6208), (129, 3136, 6080)])
@pytest.mark.parametrize("fmt", ["nvfp4", "fp8", "fp8_rows"])
def test_requantized_output(M, N, K, fmt):
    a, w, bias, res, _ = _operands(fmt, M, N, K, M + N)
    S = torch.tensor([0.002 if fmt == "nvfp4" else 0.01], device="cuda")
    alloc = qlin.alloc_nvfp4 if fmt == "nvfp4" else lambda m, k: qlin.alloc_fp8(m, k, False)
    call = qlin.qlin_linear_nvfp4 if fmt == "nvfp4" else qlin.qlin_linear_fp8
    for c0, cols in ((0, N), (64 * (N // 128), N - 64 * (N // 128))):
        q = alloc(M, cols)
        y = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
        call(a, w, bias, qlin.QLIN_ACT_GELU_TANH, res, y, S, q, c0)
        _check(y, a, w, bias, qlin.QLIN_ACT_GELU_TANH, res, (fmt, M, N, K))
        win = np.ascontiguousarray(bf16_bits(y)[:, c0:c0 + cols])
        if fmt == "nvfp4":
            codes, canon, s = nvfp4_to_host(q)
            assert s == np.float32(S.item())
            assert_requant_exact(codes, canon, win, np.float32(S.item()))
        else:
            ref, _ = oracle.quant_fp8(win, np.float32(S.item()))
            assert np.array_equal(u8(q.codes), ref) and q.scale.item() == S.item()
        q2 = alloc(M, cols)   # without the 16-bit output
        y2, _ = call(a, w, bias, qlin.QLIN_ACT_GELU_TANH, res, None, S, q2, c0)
        assert y2 is None and torch.equal(q2.codes, q.codes)


@pytest.mark.parametrize("M", [3, 300, 2048])
def test_fp8_weight_with_one_scale(M):
    # W with a tensor scale, A with one scale and with one per row
    N, K = 4096 if M == 2048 else 320, 512
    for fmt in ("fp8", "fp8_rows"):
        a, w, bias, res, _ = _operands(fmt, M, N, K, 31)
        one = qlin.qlin_quantize_act_fp8(torch.randn(N, K, device="cuda").bfloat16())
        y, _ = qlin.qlin_linear_fp8(a, one, bias, qlin.QLIN_ACT_GELU, res)
        _check(y, a, one, bias, qlin.QLIN_ACT_GELU, res, (fmt, M))


@pytest.mark.parametrize("M", [1, 5, 200, 1700, 2048])
@pytest.mark.parametrize("act", ACTS)
def test_large_and_special_values(M, act):
    # Products far out in both tails, and infinities and NaN in bias and residual,
    # stay in their columns and rows.
    N, K = 4096 if M == 2048 else 128, 64
    a = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    a[:, 0] = 1
    w = torch.zeros(N, K, dtype=torch.bfloat16, device="cuda")
    vals = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 3.0, -3.0, 12.0, -12.0, 90.0, -90.0, 1e4, -1e4, 1e20, -1e20, 3e38, -3e38],
                        device="cuda")
    w[:, 0] = vals.repeat(N // 16).to(torch.bfloat16)
    y = qlin.qlin_linear_bf16(a, w, None, act)
    v = w[:, 0].double()
    want = _act(v, act)
    want = torch.where(v < -50, torch.zeros_like(v), want) if act > 1 else want   # (64 bits: -90 e^-90 is 0 here)
    want = torch.where((v > 1e3) & torch.tensor(act > 1, device="cuda"), v, want)
    off = (y.double() - want).abs() - (2.0**-8 * want.abs() + 2.0**-18 * v.abs().clamp(max=20) * (want.abs() > 0) + 1e-18)
    assert off.max() <= 0, (act, off.max().item())
    bias = torch.zeros(N, dtype=torch.bfloat16, device="cuda")
    bias[3], bias[7] = float("inf"), float("nan")
    res = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda")
    res[M - 1, 20] = float("-inf")
    y2 = qlin.qlin_linear_bf16(a, w, bias, act, res)
    assert (y2[:, 3] == float("inf")).all() and y2[:, 7].isnan().all() and y2[M - 1, 20] == float("-inf")
    y2[:, 3], y2[:, 7], y2[M - 1, 20] = y[:, 3], y[:, 7], y[M - 1, 20]
    assert torch.equal(y2, y)


@pytest.mark.parametrize("fmt", ["nvfp4", "fp8_rows", "fp16"])
def test_repeated_and_on_another_stream(fmt):
    for M in (1, 13, 500):
        a, w, bias, res, dt = _operands(fmt, M, 576, 1088, M)
        y0 = _call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, res)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ys = [_call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, res, stream=side) for _ in range(20)]
        side.synchronize()
        assert all(torch.equal(y, y0) for y in ys)
        y, g = torch.empty_like(y0), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, res, y)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y0) and qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,N,K", [(352, 640, 12288), (555, 832, 6208), (129, 3136, 6080)])
def test_tiles_that_share_k(M, N, K, fmt):
    # eight, four and two CTAs per tile; rows and columns past the edges
    a, w, bias, res, dt = _operands(fmt, M, N, K, K)
    for b, act, r in ((None, qlin.QLIN_ACT_NONE, None), (bias, qlin.QLIN_ACT_NONE, None), (None, qlin.QLIN_ACT_NONE, res),
                      (bias, qlin.QLIN_ACT_GELU, res)):
        y = _call(fmt, a, w, b, act, r)
        _check(y, a, w, b, act, r, (fmt, M, N, K, b is None, r is None))
    # a residual in place and strided, an output that is only 16-byte aligned, other streams
    place = res.clone()
    _call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, place, place)
    assert torch.equal(place, y)
    wide = torch.zeros(M, N + 24, dtype=dt, device="cuda")
    wide[:, 8:8 + N] = res
    flat = torch.full((M * N + 16,), 5.0, dtype=dt, device="cuda")
    _call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, wide[:, 8:8 + N], flat[8:8 + M * N].view(M, N))
    assert torch.equal(flat[8:8 + M * N].view(M, N), y) and (flat[:8] == 5).all() and (flat[-8:] == 5).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ys = [_call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, res, stream=side) for _ in range(20)]
    side.synchronize()
    assert all(torch.equal(v, y) for v in ys)
    # special values stay in their rows and columns
    bias[3], bias[N - 1] = float("inf"), float("nan")
    r2 = res.clone()
    r2[M - 1, 20] = float("-inf")
    y2 = _call(fmt, a, w, bias, qlin.QLIN_ACT_GELU, r2)
    assert (y2[:, 3] == float("inf")).all() and y2[:, N - 1].isnan().all() and y2[M - 1, 20] == float("-inf")
    y2[:, 3], y2[:, N - 1], y2[M - 1, 20] = y[:, 3], y[:, N - 1], y[M - 1, 20]
    assert torch.equal(y2, y) and qlin.qlin_sync_status() == 0


def test_refusals_of_tensors():
    a = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(192, 128, dtype=torch.bfloat16, device="cuda")
    b, r = torch.zeros(192, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 192, dtype=torch.bfloat16, device="cuda")
    bad = [dict(a=a.half()), dict(w=w.t()), dict(w=w[:, :64]), dict(bias=b[:64]), dict(bias=b.float()),
           dict(residual=r[:2]), dict(residual=r.half()), dict(y=r.float()), dict(y=r[:, :64]), dict(bias=b.cpu())]
    for kw in bad:
        with pytest.raises(ValueError):
            qlin.qlin_linear_bf16(**{"a": a, "w": w, "bias": b, "residual": r, **kw})
    A, W = qlin.qlin_quantize_act_fp8(a), qlin.qlin_quantize_weight(w, qlin.QLIN_FMT_FP8)
    with pytest.raises(ValueError):
        qlin.qlin_linear_fp8(A, W, next_scale=torch.ones(1, device="cuda"))
    with pytest.raises(qlin.QlinError):
        qlin.qlin_linear_bf16(a, w, b, 9)
    with pytest.raises(qlin.QlinError):
        qlin.qlin_linear_bf16(a, w, b, 0, torch.zeros(4, 196, dtype=torch.bfloat16, device="cuda")[:, :192])
