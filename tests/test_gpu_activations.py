"""The activations of the linears at every finite 16-bit number.

A product of one element with 1 is exact, so that y is one rounding of the kernel's
activation.  The header allows 2^-13 of the value beside that rounding, and values below
2^-119 may come as zero."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

REL, SMALL = 2.0**-13, 2.0**-119


def _exact(v, act):
    if act == qlin.QLIN_ACT_RELU:
        return v.clamp(min=0)
    if act == qlin.QLIN_ACT_SILU:
        return v / (1 + torch.exp(-v))
    if act == qlin.QLIN_ACT_GELU_TANH:
        z = math.sqrt(2 / math.pi) * (v + 0.044715 * v**3)
        return v / (1 + torch.exp(-2 * z))
    return 0.5 * v * torch.special.erfc(-v / math.sqrt(2))


def _values(dtype):
    v = torch.arange(-2**15, 2**15, device="cuda").to(torch.int16).view(dtype)
    return v[torch.isfinite(v)]


@pytest.mark.parametrize("act", [qlin.QLIN_ACT_RELU, qlin.QLIN_ACT_SILU, qlin.QLIN_ACT_GELU_TANH, qlin.QLIN_ACT_GELU])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
# few tokens; tiles (of 64 to 256 columns by M and N); tiles that share K
@pytest.mark.parametrize("route,N,K,chunk", [("few", 64, 64, 1500), ("tiles", 256, 64, 70000), ("tiles", 64, 64, 70000),
                                             ("split", 64, 4160, 1200)])
def test_every_number(route, N, K, chunk, dtype, act):
    call = qlin.qlin_linear_bf16 if dtype is torch.bfloat16 else qlin.qlin_linear_fp16
    v = _values(dtype)
    w = torch.zeros(N, K, dtype=dtype, device="cuda")
    w[:, 0] = 1
    a = torch.zeros(len(v), K, dtype=dtype, device="cuda")
    a[:, 0] = v
    half, low = (2.0**-11, 2.0**-25) if dtype is torch.float16 else (2.0**-8, 2.0**-134)
    want = _exact(v.double(), act)[:, None]
    tol = half * want.abs() + (1 + half) * (REL * want.abs() + SMALL) + low
    for i in range(0, len(v), chunk):
        y = call(a[i:i + chunk], w, None, act)
        off = (y.double() - want[i:i + chunk]).abs() - tol[i:i + chunk]
        assert off.max() <= 0, (off.max().item(), v[i + off.amax(1).argmax()].item())
