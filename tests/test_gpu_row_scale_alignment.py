"""FP8 row scales that start off 16-byte boundaries (a part of a longer vector): the same
outputs as from aligned ones, in every call that reads or writes them."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu


def _shifted(q, by):
    """The operand with its scales `by` numbers into a longer vector of NaN."""
    wide = torch.full((q.rows + 8,), float("nan"), device="cuda")
    part = wide[by:by + q.scale.numel()]
    assert part.data_ptr() % 16 == 4 * by
    part.copy_(q.scale)
    return qlin.FP8Tensor(q.codes, part, q.rows, q.K, q.per_channel), wide


# few tokens, tiles of 64, 128 and 2 x 128 rows, tiles that share K
@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (20, 1344, 4160), (257, 320, 192), (552, 832, 4160), (1300, 1344, 320),
                                   (2500, 4416, 512)])
def test_products(M, N, K, by):
    g = torch.Generator(device="cuda").manual_seed(M)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, w = rnd(M, K), rnd(N, K)
    A, rows = qlin.qlin_quantize_act_fp8(x), qlin.qlin_quantize_weight(x, qlin.QLIN_FMT_FP8)
    W = qlin.qlin_quantize_weight(w, qlin.QLIN_FMT_FP8)
    W2, _ = _shifted(W, by)
    R2, _ = _shifted(rows, by)
    bias, S = rnd(N), torch.tensor([0.05], device="cuda")

    # (another tile adds in another order: products to K fp32 roundings, 2^-8 for the output's)
    def close(a, b):
        size = x.float().norm(dim=1)[:, None] * w.float().norm(dim=1)
        return ((a.float() - b.float()).abs() <= 2.0**-7 * b.float().abs() + K * 2.0**-22 * size).all()

    assert close(qlin.qlin_gemm_fp8(A, W2), qlin.qlin_gemm_fp8(A, W))
    assert close(qlin.qlin_linear_fp8(A, W2)[0], qlin.qlin_linear_fp8(A, W)[0])
    y0, y1 = (torch.empty(M, N, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q0, q1 = qlin.alloc_fp8(M, N, False), qlin.alloc_fp8(M, N, False)
    qlin.qlin_linear_fused_fp8(A, W, y0, S, q0)
    qlin.qlin_linear_fused_fp8(A, W2, y1, S, q1)
    assert close(y1, y0)

    assert torch.equal(q1.codes, (y1.float() * (1 / S)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    # with an epilogue the same kernel runs
    for a in ((rows, R2), (A, A)):
        want, _ = qlin.qlin_linear_fp8(a[0], W, bias, qlin.QLIN_ACT_SILU)
        assert torch.equal(qlin.qlin_linear_fp8(a[1], W2, bias, qlin.QLIN_ACT_SILU)[0], want)
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("by", [1, 2, 3])
@pytest.mark.parametrize("M,K", [(5, 64), (130, 3072), (3, 20480)])
def test_quantizers_that_write_them(M, K, by):
    x = torch.randn(M, K, device="cuda").bfloat16()
    for call in (lambda out: qlin.qlin_quantize_weight(x, qlin.QLIN_FMT_FP8, out),
                 lambda out: qlin.qlin_rmsnorm_fp8(x, out=out)):
        q = qlin.alloc_fp8(M, K, True)
        call(q)
        part, wide = _shifted(q, by)
        part.scale.zero_()
        part.codes = torch.zeros_like(q.codes)
        call(part)
        assert torch.equal(part.scale, q.scale) and torch.equal(part.codes, q.codes)
        assert wide[:by].isnan().all() and wide[by + M:].isnan().all()
