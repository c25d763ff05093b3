"""The block's value columns in attention's place, also after a call that was given
attention's output."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import block, qlin

pytestmark = pytest.mark.gpu

H, HEADS, F = 512, 8, 1088


@pytest.mark.parametrize("fmt", ["fp8", "nvfp4"])
@pytest.mark.parametrize("M", [3, 130])
def test_finish_without_attention_takes_the_projected_values(M, fmt):
    b = block.build_block(fmt, M, H, HEADS, F, seed=5)
    g = torch.Generator(device="cuda").manual_seed(M)
    x = torch.randn(M, H, generator=g, device="cuda").bfloat16()
    attended = torch.randn(M, H, generator=g, device="cuda").bfloat16()
    pos = torch.arange(M, device="cuda", dtype=torch.int32)
    b.calibrate(x)
    y0 = b.forward(x, pos).clone()
    b.project(x, pos)
    y1 = b.finish(x, attended).clone()
    assert not torch.equal(y1, y0)
    assert torch.equal(b.finish(x), y0)             # the values, not attention's output again
    assert torch.equal(b.finish(x, attended), y1)
    assert torch.equal(b.forward(x, pos), y0) and qlin.qlin_sync_status() == 0
