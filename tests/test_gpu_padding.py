"""The padding rows of an NVFP4 operand's scales (up to the next 128) hold anything: no
output may depend on them.  0x7F and 0xFF are E4M3 NaNs, ordinary bytes of memory that
held codes before."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu


def _padding(q):
    """The scales as [row blocks, K / 64, 32, 4, 4], and which of them are padding rows."""
    s = q.scales.view(-1, q.K // 64, 32, 4, 4)
    row = (128 * torch.arange(s.shape[0], device="cuda")[:, None, None] + 32 * torch.arange(4, device="cuda")
           + torch.arange(32, device="cuda")[:, None])
    return s, (row >= q.rows)[:, None, :, :, None].expand_as(s)


def _operands(M, N, K, fill):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    A = qlin.qlin_quantize_act_nvfp4(rnd(M, K))
    W = qlin.qlin_quantize_weight(rnd(N, K), qlin.QLIN_FMT_NVFP4)
    for q in (A, W):
        s, pad = _padding(q)
        assert pad.any() == (q.rows % 128 != 0)
        s[pad] = fill
    return A, W


# one tile and several of 128 x 64, 128 x 128 and 256 x 256; rows, columns or both past the edge
@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (77, 320, 192), (130, 128, 1088), (128, 192, 256), (1300, 1344, 320),
                                   (2500, 4416, 512)])
@pytest.mark.parametrize("fill", [0x7F, 0xFF])
def test_output_scale_of_the_chain(M, N, K, fill):
    A, W = _operands(M, N, K, 0)
    y0, q0 = qlin.qlin_linear_dynamic(A, W)
    assert torch.isfinite(q0.tensor_scale).all()
    A, W = _operands(M, N, K, fill)
    y1, q1 = qlin.qlin_linear_dynamic(A, W)
    assert torch.equal(y1, y0) and torch.equal(q1.tensor_scale, q0.tensor_scale)
    assert torch.equal(q1.codes, q0.codes)
    (s0, pad), (s1, _) = _padding(q0), _padding(q1)
    assert torch.equal(s0[~pad], s1[~pad])
    assert qlin.qlin_sync_status() == 0


# few tokens, tiles of each width, tiles that share K
@pytest.mark.parametrize("M,N,K", [(1, 64, 64), (9, 320, 1088), (77, 320, 192), (352, 320, 12288), (1300, 1344, 320),
                                   (2500, 4416, 512)])
@pytest.mark.parametrize("fill", [0x7F, 0xFF])
def test_linears(M, N, K, fill):
    scale = torch.tensor([0.002], device="cuda")
    out = []
    for f in (0, fill):
        A, W = _operands(M, N, K, f)
        plain, yq = qlin.qlin_gemm_nvfp4(A, W), qlin.alloc_nvfp4(M, N)
        y, _ = qlin.qlin_linear_nvfp4(A, W, None, qlin.QLIN_ACT_SILU, None,
                                      torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), scale, yq)
        fused = qlin.alloc_nvfp4(M, N)
        qlin.qlin_linear_fused(A, W, None, scale, fused)
        s, pad = _padding(yq)
        f_s, _ = _padding(fused)
        out.append((plain, y, yq.codes, s[~pad], fused.codes, f_s[~pad]))
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("M,K", [(1, 64), (77, 3072), (130, 1088)])
def test_norm_into_the_chain(M, K):
    # the norm's own operand, made where memory held codes: the bytes are the same each
    # time, padding among them, and so is the layer's output
    g = torch.Generator(device="cuda").manual_seed(K)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    W = qlin.qlin_quantize_weight(torch.randn(320, K, generator=g, device="cuda").bfloat16(), qlin.QLIN_FMT_NVFP4)
    scale = torch.tensor([12.0 / 2688], device="cuda")
    given, _ = qlin.qlin_rmsnorm_nvfp4(x, scale, out=qlin.alloc_nvfp4(M, K))
    y0, q0 = qlin.qlin_linear_dynamic(given, W)
    n = qlin.qlin_nvfp4_scale_bytes(M, K)
    side = torch.cuda.Stream()
    for stream in (None, side):
        with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream()):
            used = [torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        del used
        a, _ = qlin.qlin_rmsnorm_nvfp4(x, scale, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(a.scales, given.scales) and torch.equal(a.codes, given.codes)
        y1, q1 = qlin.qlin_linear_dynamic(a, W)
        assert torch.equal(y1, y0) and torch.equal(q1.tensor_scale, q0.tensor_scale) and torch.equal(q1.codes, q0.codes)
