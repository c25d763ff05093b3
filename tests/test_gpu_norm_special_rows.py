"""Rows with infinities, NaN and sums beyond fp32 in every output format of the norm, in
registers and beyond."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu


def _rows(K):
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn(4, K, generator=g, device="cuda").bfloat16()
    x[0, 37], x[0, K - 1] = float("inf"), float("-inf")
    x[1, 20] = float("nan")
    return x


# s * (1 / sqrt(infinity)) = s * 0: zeros, and NaN where s is infinite; a NaN is in the
# mean of all
@pytest.mark.parametrize("K", [64, 512, 3072, 6208, 20480])
def test_rows_with_an_infinity_or_a_nan(K):
    x = _rows(K)
    inf = x[0].isinf()
    w = torch.full((K,), 1.5, dtype=torch.bfloat16, device="cuda")
    clean = qlin.qlin_rmsnorm(x[2:], w)[0]
    for res in (None, torch.zeros_like(x)):
        y, t = qlin.qlin_rmsnorm(x, w, res)
        assert torch.equal(y[0].isnan(), inf) and (y[0][~inf] == 0).all() and y[1].isnan().all()
        assert torch.equal(y[2:], clean)
        # one static scale: the NaN code, and zeros
        q, _ = qlin.qlin_rmsnorm_fp8(x, w, res, static_scale=torch.tensor([0.01], device="cuda"))
        c = q.codes.view(torch.float8_e4m3fn).float()
        assert torch.equal(c[0].isnan(), inf) and (c[0][~inf] == 0).all() and c[1].isnan().all()
        assert torch.isfinite(c[2:]).all()
        # a scale per row: NaN, as all of the row's codes
        q, _ = qlin.qlin_rmsnorm_fp8(x, w, res)
        c = q.codes.view(torch.float8_e4m3fn).float()
        assert q.scale[:2].isnan().all() and c[:2].isnan().all()
        assert torch.isfinite(q.scale[2:]).all() and torch.isfinite(c[2:]).all()
        # NVFP4: blocks with a NaN have a NaN for their scale, other blocks zeros
        q, _ = qlin.qlin_rmsnorm_nvfp4(x, torch.tensor([0.005], device="cuda"), w, res)
        s = q.scales.view(K // 64, 32, 4, 4)[:, :4, 0].permute(1, 0, 2).reshape(4, K // 16)
        s = s.contiguous().view(torch.float8_e4m3fn).float()
        hit = inf.view(K // 16, 16).any(1)
        assert torch.equal(s[0].isnan(), hit) and (s[0][~hit] == 0).all() and s[1].isnan().all()
        assert (q.codes.view(4, K // 16, 8)[0][~hit] & 0x77 == 0).all() and torch.isfinite(s[2:]).all()


@pytest.mark.parametrize("K", [64, 3072, 20480])
def test_sums_beyond_fp32(K):
    # x + residual is an fp32 sum: two values above half of the largest make an infinity
    x = torch.full((2, K), 3e38, dtype=torch.bfloat16, device="cuda")
    x[0, 1:] = 1.0
    y, t = qlin.qlin_rmsnorm(x, None, x)
    assert t[0, 0].isinf() and (t[0, 1:] == 2).all() and t[1].isinf().all()
    assert y[0, 0].isnan() and (y[0, 1:] == 0).all() and y[1].isnan().all()
    # the largest finite sums go through scaled squares
    big = torch.full((1, K), 1.5e38, dtype=torch.bfloat16, device="cuda")
    y, t = qlin.qlin_rmsnorm(big, None, big)
    assert torch.isfinite(t.float()).all() and (y == 1).all()
