"""The block-scaled FP8 quantizer bit for bit against its formula, and the linear of its
operands against the formula in 64 bits.

Linear's tolerance, before the rounding to bf16: a block's products are summed in fp32 steps
of at least 16 elements, and each block's sum is scaled and added with a rounding for the
scale and one for the sum; no running sum exceeds ||a|| ||w|| of the scaled operands, so
(K / 16 + K / 64 + 8) 2^-23 ||a|| ||w||.  The activations' slope is at most 1.13;
exponentials, quotients and the additions keep 2^-18 of the values they meet."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

ACTS = [qlin.QLIN_ACT_NONE, qlin.QLIN_ACT_RELU, qlin.QLIN_ACT_SILU, qlin.QLIN_ACT_GELU_TANH, qlin.QLIN_ACT_GELU]


def _blocks(x, br):
    """[row blocks, br, K blocks, 128], filled with zeros."""
    r, k = x.shape
    p = torch.nn.functional.pad(x, (0, -k % 128, 0, -r % br))
    return p.view(-1, br, p.shape[1] // 128, 128)


def _quantized(x, br):
    """(codes uint8, scales [K blocks, row blocks]) by the formula, on the CPU in fp32."""
    b = _blocks(x.float().cpu(), br)
    amax = b.abs().amax((1, 3))
    S = torch.where(amax == 0, torch.ones(()), amax / 448)
    enc = 1 / S
    enc = torch.where(torch.isinf(enc), torch.full((), torch.finfo(torch.float32).max), enc)
    v = (b * enc[:, None, :, None]).reshape(-1, b.shape[2] * 128)[:x.shape[0], :x.shape[1]]
    return v.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), S.t().contiguous()


def _normal(*shape, seed, dtype=torch.bfloat16, sigma=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * sigma).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,K,br,wide,first", [
    (1, 64, 1, 0, 0), (1, 64, 128, 0, 0), (3, 192, 1, 8, 0), (4, 128, 1, 0, 0), (5, 1088, 1, 24, 8), (129, 320, 128, 8, 8),
    (127, 128, 128, 0, 0), (1000, 640, 1, 0, 0), (333, 1088, 128, 64, 16), (4608, 3072, 1, 0, 0), (2, 12288, 1, 0, 0)])
def test_quantizer(rows, K, br, wide, first, dtype):
    base = _normal(rows, first + K + wide, seed=rows + K, dtype=dtype)
    x = base[:, first:first + K]
    x[rows // 2, : min(K, 128)] = 0
    x[rows - 1] *= 2.0**-8
    q = qlin.qlin_quantize_fp8_block(x, br)
    codes, S = _quantized(x, br)
    assert torch.equal(q.scales.cpu(), S)
    assert torch.equal(q.codes.cpu(), codes)
    # nothing outside the operand
    out = qlin.alloc_fp8_block(rows, K, br)
    buf = torch.full((rows * K + 256,), 7, dtype=torch.uint8, device="cuda")
    sbuf = torch.full((out.scales.numel() + 8,), -3.0, device="cuda")
    out.codes, out.scales = buf[128:128 + rows * K].view(rows, K), sbuf[4:4 + out.scales.numel()].view(out.scales.shape)
    qlin.qlin_quantize_fp8_block(x, out=out)
    assert torch.equal(out.codes, q.codes) and torch.equal(out.scales, q.scales)
    assert (buf[:128] == 7).all() and (buf[128 + rows * K:] == 7).all()
    assert (sbuf[:4] == -3).all() and (sbuf[-4:] == -3).all()
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("br", [1, 128])
def test_quantizer_extremes(br):
    # the smallest and largest values, signed zeros, and blocks with NaN and infinities
    x = _normal(256, 512, seed=1)
    x[0, 0:128] = 1e-40
    x[1, 0:128] = -0.0
    x[2, 0:128] = torch.finfo(torch.bfloat16).max
    x[3, 130] = 9.2e-41
    q = qlin.qlin_quantize_fp8_block(x, br)
    codes, S = _quantized(x, br)
    assert torch.equal(q.scales.cpu(), S) and torch.equal(q.codes.cpu(), codes)
    x[5, 256 + 7], x[200, 384 + 3] = float("nan"), float("inf")
    q = qlin.qlin_quantize_fp8_block(x, br)
    v = q.codes.view(torch.float8_e4m3fn).float()
    r = slice(5, 6) if br == 1 else slice(0, 128)
    assert q.scales[2, 5 // br].isnan() and v[r, 256:384].isnan().all()
    r = slice(200, 201) if br == 1 else slice(128, 256)
    assert q.scales[3, 200 // br] == float("inf") and v[200, 387].isnan() and (v[r, 384:512].nan_to_num(0) == 0).all()
    assert not v[:, :256].isnan().any() and not q.scales[:2].isnan().any()


def _operand(M, K, br, seed, sigma=1.0):
    x = _normal(M, K, seed=seed, sigma=sigma)
    x[:, seed % K] *= 20                       # an outlier channel
    return qlin.qlin_quantize_fp8_block(x, br)


def _values(q):
    r = torch.arange(q.rows, device="cuda") // q.block_rows
    k = torch.arange(q.K, device="cuda") // 128
    return q.codes.view(torch.float8_e4m3fn).double() * q.scales.double()[k[None], r[:, None]]


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


def _check(y, A, W, bias, act, residual):
    a, w = _values(A), _values(W)
    v = a @ w.t()
    tol = (A.K / 16 + A.K / 64 + 8) * 2.0**-23 * torch.outer(a.norm(dim=1), w.norm(dim=1))
    if bias is not None:
        v = v + bias.double()
        tol = tol + 2.0**-18 * bias.double().abs()
    want = _act(v, act)
    tol = 1.13 * tol + 2.0**-18 * v.abs()
    if residual is not None:
        want = want + residual.double()
    tol = tol + 2.0**-18 * want.abs()
    off = (y.double() - want).abs() - (tol + 2.0**-8 * (want.abs() + tol) + 2.0**-119)
    assert off.max() <= 0, (off.max().item(), torch.nonzero(off > 0)[:4].tolist())


SHAPES = [(1, 64, 64), (1, 192, 12288), (2, 128, 128), (7, 320, 192), (16, 3072, 1088), (17, 2112, 1088), (33, 64, 4096),
          (700, 192, 12288), (700, 1024, 4096), (129, 256, 64), (128, 128, 128), (257, 320, 320), (500, 1088, 2112), (1333, 2112, 1088), (2000, 5120, 192),
          (3000, 3008, 448), (4608, 12288, 256)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(M, N, K):
    A, W = _operand(M, K, 1, 3 * M + N), _operand(N, K, 128, N + K, 1 / math.sqrt(K))
    _check(qlin.qlin_linear_fp8_block(A, W), A, W, None, qlin.QLIN_ACT_NONE, None)
    bias, wide = _normal(N, seed=5), _normal(M, N + 16, seed=6)
    for i, act in enumerate(ACTS):
        b = bias if i != 2 else None
        res = None if i % 2 else wide[:, :N] if i else wide[:, 8:N + 8]
        _check(qlin.qlin_linear_fp8_block(A, W, b, act, res), A, W, b, act, res)
    # over the residual, nothing behind y, equal calls
    buf = torch.full((M * N + 512,), 3.0, dtype=torch.bfloat16, device="cuda")
    y = buf[256 + 8:256 + 8 + M * N].view(M, N)
    y.copy_(wide[:, :N])
    res = y.clone()
    qlin.qlin_linear_fp8_block(A, W, bias, qlin.QLIN_ACT_SILU, y, y)
    assert torch.equal(y, qlin.qlin_linear_fp8_block(A, W, bias, qlin.QLIN_ACT_SILU, res))
    assert (buf[:264] == 3).all() and (buf[264 + M * N:] == 3).all()
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("M", [1, 40, 300, 3000])
def test_linear_dyadic(M):
    # small integers and powers of two as scales: every product and sum is exact
    N, K = 1024, 448
    g = torch.Generator(device="cuda").manual_seed(M)
    ints = lambda r: torch.randint(-8, 9, (r, K), generator=g, device="cuda").float().to(torch.float8_e4m3fn)  # noqa: E731
    powers = lambda *s: 2.0 ** torch.randint(-2, 3, s, generator=g, device="cuda").float()  # noqa: E731
    A = qlin.FP8BlockTensor(ints(M).view(torch.uint8), powers(4, M), M, K, 1)
    W = qlin.FP8BlockTensor(ints(N).view(torch.uint8), powers(4, N // 128), N, K, 128)
    y = qlin.qlin_linear_fp8_block(A, W)
    assert torch.equal(y, (_values(A) @ _values(W).t()).to(torch.bfloat16))


@pytest.mark.parametrize("M", [5, 600])
def test_nan_and_infinite_scales_stay_in_their_rows(M):
    N, K = 256, 384
    A, W = _operand(M, K, 1, 1), _operand(N, K, 128, 2)
    clean = qlin.qlin_linear_fp8_block(A, W)
    A.scales[1, 3] = float("nan")
    W.scales[2, 1] = float("nan")
    y = qlin.qlin_linear_fp8_block(A, W)
    assert y[3].isnan().all() and y[:, 128:].isnan().all()
    keep = torch.arange(M, device="cuda") != 3
    assert torch.equal(y[keep, :128], clean[keep, :128])


@pytest.mark.parametrize("M,N", [(3, 64), (700, 1024)])
def test_linear_on_a_stream_and_in_a_graph(M, N):
    K = 640
    A, W = _operand(M, K, 1, 1), _operand(N, K, 128, 2)
    want = qlin.qlin_linear_fp8_block(A, W)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = qlin.qlin_linear_fp8_block(A, W, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
    x = _normal(M, K, seed=9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qlin.qlin_quantize_fp8_block(x, out=A)
        qlin.qlin_linear_fp8_block(A, W, y=y)
    for seed in (10, 11):
        x.copy_(_normal(M, K, seed=seed))
        graph.replay()
        eager = qlin.qlin_linear_fp8_block(qlin.qlin_quantize_fp8_block(x), W)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)
