"""FP8 codes of the norm bit for bit as the header states them, for rows in registers and
beyond."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

LENGTHS = [64, 1088, 3072, 6208, 16384, 20480, 49152]


def _codes(v):
    """E4M3 codes of fp32 values, saturating."""
    return v.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("K", LENGTHS)
def test_codes_of_row_scales(K, dtype, weight):
    # code = E4M3((s * r) * weight), r = 448 / max |s * weight|, in fp32 one operation at a time
    M = 33
    g = torch.Generator(device="cuda").manual_seed(K)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, res = (4 * rnd(M, K)).to(dtype), rnd(M, K).to(dtype)
    w = (1 + 0.2 * rnd(K)).to(dtype) if weight else None
    q, _ = qlin.qlin_rmsnorm_fp8(x, w, res)
    s = x.cpu().float() + res.cpu().float()
    f = w.cpu().float() if weight else torch.ones(K)
    r = torch.from_numpy(np.float32(448) / (s * f).abs().amax(1, keepdim=True).numpy())
    assert torch.equal(q.codes.cpu(), _codes((s * r) * f))


@pytest.mark.parametrize("K", LENGTHS)
def test_ties(K):
    # max |t| = 28: 448 / 28 is 16, t * 16 is exact, and half of the odd t above 16 lie
    # half way between two codes; powers of two as weights
    i = torch.arange(3 * K, device="cuda").view(3, K)
    w = torch.tensor([1.0, 2.0, 0.5], device="cuda")[torch.arange(K, device="cuda") % 3]
    t = ((i * 13) % 57 - 28).float()
    t[:, 0] = 28
    x = (t / w).bfloat16()
    assert torch.equal(x.float() * w, t)
    q, _ = qlin.qlin_rmsnorm_fp8(x, w.bfloat16())
    assert torch.equal(q.codes, _codes(16 * t))
