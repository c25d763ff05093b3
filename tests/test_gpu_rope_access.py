"""The bits of a rotated value depend on the value, its position and its place in the head
alone: whatever strides and alignments choose, wide accesses or single elements."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,R", [(191, 12, 512, 424), (290, 49, 128, 80), (700, 24, 128, 128), (130, 50, 1000, 240),
                                     (300, 40, 24, 8)])
def test_bits(T, H, D, R, layout, dtype, inverse):
    g = torch.Generator(device="cuda").manual_seed(D + R)
    x = torch.randn(T, H, D, generator=g, device="cuda").to(dtype)
    pos = torch.randint(-100000, 100000, (T,), generator=g, device="cuda")
    plan = qlin.rope_plan(R, layout=layout)
    y = qlin.qlin_rope(x, pos, plan, inverse=inverse)
    for first, wide in ((0, 8), (8, 0), (0, 3), (1, 0), (4, 4)):
        flat = torch.zeros(T, first + H * D + wide, dtype=dtype, device="cuda")
        flat[:, first:first + H * D] = x.view(T, H * D)
        part = flat[:, first:first + H * D].view(T, H, D)
        assert torch.equal(qlin.qlin_rope(part, pos, plan, inverse=inverse), y), (first, wide)
        assert torch.equal(qlin.qlin_rope(part, pos, plan, part, inverse=inverse), y), (first, wide)
