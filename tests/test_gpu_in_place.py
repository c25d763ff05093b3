"""In-place calls that are allowed: one row or one head of any stride, y over the
residual, negative strides."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K", [(1, 512), (5, 3072), (3, 20480)])
def test_norm(M, K):
    g = torch.Generator(device="cuda").manual_seed(K)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, r, w = rnd(M, K), rnd(M, K), rnd(K)
    y0, t0 = qlin.qlin_rmsnorm(x, w, r)
    over = r.clone()
    y1, t1 = qlin.qlin_rmsnorm(x, w, over, y=over)
    assert y1 is over and torch.equal(y1, y0) and torch.equal(t1, t0)
    wide = torch.zeros(M, 3 * K, dtype=x.dtype, device="cuda")
    wide[:, K:2 * K] = x
    part = wide[:, K:2 * K]
    if M == 1:   # a single row has no stride
        qlin.qlin_rmsnorm(part, w, r, y=part)
        assert torch.equal(part, y0)
    else:
        with pytest.raises(ValueError):
            qlin.qlin_rmsnorm(part, w, r, y=part)
    with pytest.raises(qlin.QlinError):
        qlin.qlin_rmsnorm(x, w, r, sum_out=over, y=over)


def test_rotary_heads():
    x = torch.randn(6, 4, 64, device="cuda").bfloat16()
    pos, plan = torch.arange(6, device="cuda"), qlin.rope_plan(64)
    y = qlin.qlin_rope(x, pos, plan)
    one = torch.empty(6, 1, 64, dtype=x.dtype, device="cuda").expand(6, 1, 64)
    assert torch.equal(qlin.qlin_rope(x[:, :1], pos, plan, one), y[:, :1])
    for out in (torch.empty(6, 1, 64, dtype=x.dtype, device="cuda").expand(6, 4, 64),
                torch.empty(1, 4, 64, dtype=x.dtype, device="cuda").expand(6, 4, 64)):
        with pytest.raises(qlin.QlinError):
            qlin.qlin_rope(x, pos, plan, out)
    same = x[:, :1].expand(6, 4, 64)     # an expanded input is fine
    assert torch.equal(qlin.qlin_rope(same, pos, plan), y[:, :1].expand(6, 4, 64))
    with pytest.raises(qlin.QlinError):
        qlin.qlin_rope(same, pos, plan, same)
