"""Tiles whose warps store odd numbers of boxes, several tiles per CTA: every output of
repeated calls against exact products.  Operands of -1, 0 and 1 with K <= 192 and a
residual of small integers: every sum is an integer below 256, exact in every format."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_staging_boxes import NARROW_SIZES, WIDE_SIZES

pytestmark = pytest.mark.gpu

CALLS = 30


def _signs(rows, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-1, 2, (rows, K), generator=g, device="cuda")


def _fp8(v):
    codes = v.float().to(torch.float8_e4m3fn).view(torch.uint8)
    return qlin.FP8Tensor(codes, torch.ones(1, device="cuda"), v.shape[0], v.shape[1], 0)


def _nvfp4(v):
    q = qlin.alloc_nvfp4(*v.shape)
    c = torch.where(v > 0, 2, torch.where(v < 0, 10, 0)).to(torch.uint8)   # e2m1 1, -1, 0
    q.codes.copy_(c[:, ::2] | (c[:, 1::2] << 4))
    q.scales.fill_(0x38)   # E4M3 1
    q.tensor_scale.fill_(1.0)
    return q


def _repeat(call, want):
    for _ in range(CALLS):
        y = torch.full(want.shape, float("nan"), dtype=want.dtype, device="cuda")
        call(y)
        assert torch.equal(y, want)
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,N,K", WIDE_SIZES)
def test_three_stores_per_tile(M, N, K, dtype, residual):
    a, w = _signs(M, K, 1), _signs(N, K, 2)
    r = torch.randint(-9, 10, (M, N), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    exact = a.float() @ w.float().t() + (r if residual else 0)
    assert exact.abs().max() < 256
    a, w, r = a.to(dtype), w.to(dtype), r.to(dtype)
    bias = torch.zeros(N, dtype=dtype, device="cuda")
    call = qlin.qlin_linear_bf16 if dtype is torch.bfloat16 else qlin.qlin_linear_fp16
    _repeat(lambda y: call(a, w, bias, residual=r if residual else None, y=y), exact.to(dtype))


@pytest.mark.parametrize("fmt", ["fp8", "nvfp4"])
@pytest.mark.parametrize("M,N,K", NARROW_SIZES)
def test_one_store_per_tile(M, N, K, fmt):
    a, w = _signs(M, K, 4), _signs(N, K, 5)
    want = (a.float() @ w.float().t()).bfloat16()
    make, plain, linear = ((_fp8, qlin.qlin_gemm_fp8, qlin.qlin_linear_fp8) if fmt == "fp8"
                           else (_nvfp4, qlin.qlin_gemm_nvfp4, qlin.qlin_linear_nvfp4))
    A, W = make(a), make(w)
    bias = torch.zeros(N, dtype=torch.bfloat16, device="cuda")
    _repeat(lambda y: plain(A, W, y), want)
    _repeat(lambda y: linear(A, W, bias, y=y), want)
