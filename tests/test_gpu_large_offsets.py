"""Rows whose offsets pass 32 bits, in elements and in bytes: views of a buffer of 2^32
bytes and more, against the same call on compact copies, bit for bit."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def far():
    """A [5, 2^30] bf16 matrix (10 GB): row 2 starts at element 2^31, byte 2^32."""
    buf = torch.empty(5, 1 << 30, dtype=torch.bfloat16, device="cuda")
    yield buf
    del buf
    torch.cuda.empty_cache()


def test_norm(far):
    K = 1024
    x, r, s = far[:, :K], far[:, 4096:4096 + K], far[:, 8192:8192 + K]
    xc, rc = torch.randn(5, K, device="cuda").bfloat16(), torch.randn(5, K, device="cuda").bfloat16()
    x.copy_(xc)
    r.copy_(rc)
    w = torch.randn(K, device="cuda").bfloat16()
    q0, s0 = qlin.qlin_rmsnorm_fp8(xc, w, rc)
    q1, _ = qlin.qlin_rmsnorm_fp8(x, w, r, sum_out=s)
    assert torch.equal(q0.codes, q1.codes) and torch.equal(q0.scale, q1.scale) and torch.equal(s, s0)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("shift", [0, 1])     # 16-byte accesses, and single elements
def test_rope(far, layout, shift):
    T, H, D = 5, 3, 64
    c = torch.randn(T, H, D, device="cuda").bfloat16()
    pos = torch.arange(T, device="cuda") * 1001
    plan = qlin.rope_plan(48, layout=layout)
    want = qlin.qlin_rope(c, pos, plan)
    # far tokens, and far heads
    x = far[:, 16384 + shift:16384 + shift + H * D].view(T, H, D)
    x.copy_(c)
    assert torch.equal(qlin.qlin_rope(x, pos, plan, x), want)
    h = far[:, 32768 + shift:32768 + shift + T * D].view(5, T, D)[:H].transpose(0, 1)
    h.copy_(c)
    assert torch.equal(qlin.qlin_rope(h, pos, plan), want)


@pytest.mark.parametrize("M", [5, 300])
def test_linear(far, M):
    N, K = 192, 256
    a, w = torch.randn(M, K, device="cuda").bfloat16(), torch.randn(N, K, device="cuda").bfloat16()
    res = torch.randn(M, N, device="cuda").bfloat16()
    want = qlin.qlin_linear_bf16(a, w, None, qlin.QLIN_ACT_SILU, res)
    stride = (far.numel() // M) // 8 * 8
    rows = far.view(-1)[:M * stride].view(M, stride)
    af, rf = rows[:, 1024:1024 + K], rows[:, 2048:2048 + N]
    af.copy_(a)
    rf.copy_(res)
    assert torch.equal(qlin.qlin_linear_bf16(af, w, None, qlin.QLIN_ACT_SILU, rf), want)
    assert qlin.qlin_sync_status() == 0
