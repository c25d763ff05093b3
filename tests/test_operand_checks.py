"""Quantized operands and scales that a kernel cannot read are refused in Python: their
addresses alone say nothing of memory or type."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin


def _fp8(rows, K, device, per_channel=True):
    return qlin.FP8Tensor(torch.zeros(rows, K, dtype=torch.uint8, device=device),
                          torch.ones(rows if per_channel else 1, device=device), rows, K, 1 if per_channel else 0)


def _nvfp4(rows, K, device):
    n = (rows + 127) // 128 * (K // 64) * 512
    return qlin.NVFP4Tensor(torch.zeros(rows, K // 2, dtype=torch.uint8, device=device),
                            torch.zeros(n, dtype=torch.uint8, device=device), torch.ones(1, device=device), rows, K)


def test_operands_of_the_host():
    with pytest.raises(ValueError, match="CUDA"):
        qlin.qlin_linear_fp8(_fp8(4, 128, "cpu"), _fp8(64, 128, "cpu"))
    with pytest.raises(ValueError, match="CUDA"):
        qlin.qlin_linear_nvfp4(_nvfp4(4, 128, "cpu"), _nvfp4(64, 128, "cpu"))


@pytest.mark.gpu
def test_operands_of_two_devices():
    a8, w8, a4, w4 = _fp8(4, 128, "cuda"), _fp8(64, 128, "cuda"), _nvfp4(4, 128, "cuda"), _nvfp4(64, 128, "cuda")
    part8 = qlin.FP8Tensor(w8.codes, w8.scale.cpu(), 64, 128, 1)
    part4 = qlin.NVFP4Tensor(w4.codes, w4.scales, w4.tensor_scale.cpu(), 64, 128)
    blocks = qlin.NVFP4Tensor(a4.codes, a4.scales.cpu(), a4.tensor_scale, 4, 128)
    S = torch.ones(1, device="cuda")
    for A, W in ((a8, _fp8(64, 128, "cpu")), (a8, part8)):
        with pytest.raises(ValueError, match="W"):
            qlin.qlin_linear_fp8(A, W)
    with pytest.raises(ValueError, match="W"):
        qlin.qlin_linear_nvfp4(a4, part4)
    with pytest.raises(ValueError, match="A"):
        qlin.qlin_linear_nvfp4(blocks, w4)
    with pytest.raises(ValueError, match="y_q"):
        qlin.qlin_linear_fp8(a8, w8, next_scale=S, y_q=_fp8(4, 64, "cpu", False))
    x = torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="out"):
        qlin.qlin_rmsnorm_fp8(x, out=_fp8(4, 128, "cpu"))
    with pytest.raises(ValueError, match="out"):
        qlin.qlin_rmsnorm_nvfp4(x, S, out=blocks)


@pytest.mark.gpu
@pytest.mark.parametrize("make", [lambda: torch.ones(1), lambda: torch.ones(1, dtype=torch.float64, device="cuda"),
                                  lambda: torch.ones(1, dtype=torch.bfloat16, device="cuda"),
                                  lambda: torch.ones(0, device="cuda")])
def test_scales(make):
    bad, x = make(), torch.zeros(4, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="static_scale"):
        qlin.qlin_rmsnorm_fp8(x, static_scale=bad)
    with pytest.raises(ValueError, match="static_scale"):
        qlin.qlin_rmsnorm_nvfp4(x, bad)
    with pytest.raises(ValueError, match="next_scale"):
        qlin.qlin_linear_fp8(_fp8(4, 128, "cuda"), _fp8(64, 128, "cuda"), next_scale=bad, y_q=_fp8(4, 64, "cuda", False))
    with pytest.raises(ValueError, match="next_scale"):
        qlin.qlin_linear_nvfp4(_nvfp4(4, 128, "cuda"), _nvfp4(64, 128, "cuda"), next_scale=bad, y_q=_nvfp4(4, 64, "cuda"))


@pytest.mark.gpu
def test_scales_that_are_taken():
    # a scalar, a part of a vector, an address
    x = torch.randn(4, 128, device="cuda").bfloat16()
    s = torch.tensor([3.0, 0.05, 0.05], device="cuda")
    want, _ = qlin.qlin_rmsnorm_fp8(x, static_scale=torch.tensor([0.05], device="cuda"))
    for scale in (torch.tensor(0.05, device="cuda"), s[1:2], s[1:], s[1:].data_ptr()):
        got, _ = qlin.qlin_rmsnorm_fp8(x, static_scale=scale)
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scale, want.scale)
