"""The residual addition and norm against its formula in 64 bits.

Tolerances.  s = x + r is one fp32 rounding (2^-24); a sum of K <= 49152 squares in
chains of at most 200 terms and a tree has a relative error below 2^-16, half of it
in the root; the root, the quotient, the products and the weight add 2^-21.  So n is
right to REL = 2^-16, then rounded once to the output's format."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

REL = 2.0**-16
UNIT = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}      # half a last place
LEAST = {torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}   # and of the smallest numbers
DTYPES = [torch.bfloat16, torch.float16]
# one unit, odd counts of units, a row per warp and per CTA, and rows beyond registers
SHAPES = [(1, 64), (1, 3072), (3, 192), (33, 1088), (257, 2560), (5, 4160), (2, 12288), (3, 20480), (2, 49152),
          (1300, 320), (700, 1024)]


def _inputs(M, K, dtype, seed, residual=True, weight=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = rnd(M, K)
    x[:, ::max(1, K // 7)] *= 20
    return (x.to(dtype), rnd(M, K).to(dtype) if residual else None,
            (1 + 0.2 * rnd(K)).to(dtype) if weight else None)


def _exact(x, r, w, eps):
    s = x.double() if r is None else x.double() + r.double()
    n = s / torch.sqrt(s.square().mean(1, keepdim=True) + eps)
    return s, n if w is None else n * w.double()


def _check16(y, want, dtype, what):
    off = (y.double() - want).abs() - ((UNIT[dtype] + REL) * want.abs() + LEAST[dtype])
    assert off.max() <= 0, (what, off.max().item())


def _check_fp8(codes, t, what):
    """Codes against the exact quotients t: nearest E4M3 value, up to REL of t."""
    c = codes.view(torch.float8_e4m3fn).double()
    t = t.clamp(-448, 448)
    a = t.abs().clamp(min=2.0**-6)
    half = torch.exp2(torch.floor(torch.log2(a)) - 4)
    off = (c - t).abs() - (half + 2 * REL * t.abs())
    assert off.max() <= 0, (what, off.max().item())


def _check_nvfp4(q, n, S, what):
    import oracle
    M, K = n.shape
    canon = oracle.unswizzle_scales(q.scales.cpu().numpy(), M, K)
    s = torch.from_numpy(np.ascontiguousarray(canon)).cuda().view(torch.float8_e4m3fn).double()
    t = (n.view(M, K // 16, 16).abs().amax(2) / 6 / S).clamp(max=448)
    half = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0**-6))) - 4)
    off = (s - t).abs() - (half + 2 * REL * t)
    assert off.max() <= 0, (what, "scales", off.max().item())
    grid = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
    c = torch.stack([grid[(q.codes & 15).long()], grid[(q.codes >> 4).long()]], 2).view(M, K // 16, 16)
    v = n.view(M, K // 16, 16) / (S * torch.where(s > 0, s, torch.ones_like(s)))[..., None]
    v = torch.where(s[..., None] > 0, v, torch.zeros_like(v)).clamp(-6, 6)
    a = v.abs()
    half = torch.where(a <= 2, 0.25, torch.where(a <= 4, 0.5, 1.0))
    off = (c - v).abs() - (half + 4 * REL * a.clamp(min=1))
    assert off.max() <= 0, (what, "codes", off.max().item())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", SHAPES)
def test_every_output(M, K, dtype):
    x, r, w = _inputs(M, K, dtype, M + K)
    s, n = _exact(x, r, w, 1e-6)
    y, t = qlin.qlin_rmsnorm(x, w, r)
    _check16(t, s, dtype, "sum")
    _check16(y, n, dtype, "y")
    q, t2 = qlin.qlin_rmsnorm_fp8(x, w, r)
    assert torch.equal(t, t2)
    S = n.abs().amax(1) / 448
    assert ((q.scale.double() - S).abs() <= 2 * REL * S).all()
    _check_fp8(q.codes, n / S[:, None], "fp8 rows")
    sc = torch.tensor([8.0 / 448], device="cuda")   # values beyond 8 saturate
    q, _ = qlin.qlin_rmsnorm_fp8(x, w, r, static_scale=sc)
    assert q.scale.item() == sc.item() and q.per_channel == 0
    _check_fp8(q.codes, n / sc.double(), "fp8")
    sc = torch.tensor([12.0 / 2688], device="cuda")
    q, t3 = qlin.qlin_rmsnorm_nvfp4(x, sc, w, r)
    assert q.tensor_scale.item() == sc.item() and torch.equal(t, t3)
    _check_nvfp4(q, n, sc.double(), "nvfp4")
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("residual,weight", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("M,K", [(7, 512), (3, 6208)])
def test_parts_left_out(M, K, residual, weight):
    x, r, w = _inputs(M, K, torch.bfloat16, 5, residual, weight)
    s, n = _exact(x, r, w, 1e-3)
    y, t = qlin.qlin_rmsnorm(x, w, r, eps=1e-3)
    assert (t is None) == (not residual)
    _check16(y, n, torch.bfloat16, "y")
    q, _ = qlin.qlin_rmsnorm_fp8(x, w, r, eps=1e-3)
    _check_fp8(q.codes, n / (n.abs().amax(1, keepdim=True) / 448), "fp8 rows")


@pytest.mark.parametrize("M,K", [(33, 1088), (4, 12288), (2, 20480)])
def test_strided_rows_and_in_place(M, K):
    dtype = torch.bfloat16
    x, r, w = _inputs(M, K, dtype, 9)
    y0, t0 = qlin.qlin_rmsnorm(x, w, r)
    wide = [torch.full((M, K + 72), 7.0, dtype=dtype, device="cuda") for _ in range(3)]
    xs, rs, ss = (v[:, 8:8 + K] for v in wide)
    xs.copy_(x)
    rs.copy_(r)
    y1, t1 = qlin.qlin_rmsnorm(xs, w, rs, sum_out=ss)
    assert torch.equal(y0, y1) and torch.equal(t0, ss) and t1 is ss
    for v in wide:   # nothing beside the rows
        assert (v[:, :8] == 7).all() and (v[:, 8 + K:] == 7).all()
    # the stream updated in place: over x, over the residual; y over x
    xa, ra = x.clone(), r.clone()
    q0, _ = qlin.qlin_rmsnorm_fp8(x, w, r)
    q1, _ = qlin.qlin_rmsnorm_fp8(xa, w, ra, sum_out=xa)
    assert torch.equal(xa, t0) and torch.equal(q0.codes, q1.codes) and torch.equal(q0.scale, q1.scale)
    y2, _ = qlin.qlin_rmsnorm(x, w, ra, sum_out=ra)
    assert torch.equal(ra, t0) and torch.equal(y2, y0)
    xa = x.clone()
    y3, _ = qlin.qlin_rmsnorm(xa, w, r, y=xa)
    assert torch.equal(xa, y0)


@pytest.mark.parametrize("K", [512, 6208, 20480])
def test_extreme_rows(K):
    x, _, w = _inputs(8, K, torch.bfloat16, 3, residual=False)
    x[0] = 0                                    # scale 1, codes 0
    x[1, 5] = float("nan")
    x[2, 7] = float("inf")
    x[3] = x[3] * 2.0**100                      # squares overflow fp32
    x[4] = 3e38                                 # and so do the sum's terms by far
    x[5] = x[5] * 2.0**-100                     # squares vanish beside eps
    s, n = _exact(x, None, w, 1e-6)
    y, _ = qlin.qlin_rmsnorm(x, w)
    for i in (1, 2):
        assert y[i].isnan().any()
    assert y[1].isnan().all()                   # a NaN poisons its row
    ok = [0, 3, 4, 5, 6, 7]
    _check16(y[ok], n[ok], torch.bfloat16, "y")
    q, _ = qlin.qlin_rmsnorm_fp8(x, w)
    assert q.scale[0].item() == 1.0 and (q.codes[0] == 0).all()
    assert q.scale[1].isnan() and q.scale[2].isnan()
    S = n[ok].abs().amax(1) / 448
    good = S > 0
    assert ((q.scale[ok].double() - S)[good].abs() <= 2 * REL * S[good]).all()
    rows = [i for i in ok if i != 0 and i != 5]
    _check_fp8(q.codes[rows], n[rows] / (n[rows].abs().amax(1, keepdim=True) / 448), "fp8 rows")
    # the largest sum of two values, in scaled squares as well
    big = torch.full((1, K), 3e38, dtype=torch.bfloat16, device="cuda")
    y, t = qlin.qlin_rmsnorm(big, None, -big)
    assert (y == 0).all() and (t == 0).all()


@pytest.mark.parametrize("K", [64, 1088, 3072, 20480])
def test_row_scales_of_weighted_rows_near_the_largest_number(K):
    # max |x weight| beyond 2^126, and rows whose codes are exact
    x = torch.full((3, K), 1e17, dtype=torch.bfloat16, device="cuda")
    x[:, ::3] *= -0.5
    w = torch.full((K,), 1.5e21, dtype=torch.bfloat16, device="cuda")
    q, _ = qlin.qlin_rmsnorm_fp8(x, w)
    _, n = _exact(x, None, w, 1e-6)
    S = n.abs().amax(1) / 448
    assert ((q.scale.double() - S).abs() <= 2 * REL * S).all()
    _check_fp8(q.codes, n / q.scale.double()[:, None], K)
    v = torch.arange(-14, 15, device="cuda").float()[torch.arange(3 * K, device="cuda") % 29].view(3, K).to(torch.bfloat16)
    q, _ = qlin.qlin_rmsnorm_fp8(v)
    assert torch.equal(q.codes.view(torch.float8_e4m3fn).float(), v.float() * 32)


def test_repeated_and_on_another_stream():
    x, r, w = _inputs(513, 2560, torch.bfloat16, 4)
    q0, t0 = qlin.qlin_rmsnorm_fp8(x, w, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [qlin.qlin_rmsnorm_fp8(x, w, r, stream=side) for _ in range(20)]
    side.synchronize()
    for q, t in outs:
        assert torch.equal(q.codes, q0.codes) and torch.equal(q.scale, q0.scale) and torch.equal(t, t0)
    g = torch.cuda.CUDAGraph()
    out, s = qlin.alloc_fp8(513, 2560, True), torch.empty_like(x)
    with torch.cuda.graph(g):
        qlin.qlin_rmsnorm_fp8(x, w, r, sum_out=s, out=out)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.codes, q0.codes) and torch.equal(s, t0)


def test_refusals_of_tensors():
    x, r, w = _inputs(4, 256, torch.bfloat16, 1)
    bad = [dict(x=x.float()), dict(x=x.t()), dict(x=x[0]), dict(residual=r[:3]), dict(residual=r.half()),
           dict(weight=w[:128]), dict(weight=w.half()), dict(sum_out=torch.empty(4, 128, dtype=x.dtype, device="cuda")),
           dict(residual=None, sum_out=x), dict(y=torch.empty(4, 256, device="cuda")), dict(y=r.t().contiguous().t())]
    for kw in bad:
        args = {"x": x, "weight": w, "residual": r, **kw}
        with pytest.raises(ValueError):
            qlin.qlin_rmsnorm(**args)
    with pytest.raises(qlin.QlinError):
        qlin.qlin_rmsnorm(torch.zeros(2, 96, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(qlin.QlinError):
        qlin.qlin_rmsnorm(torch.zeros(2, 72, dtype=torch.bfloat16, device="cuda")[:, 4:68])
    with pytest.raises(qlin.QlinError):
        qlin.qlin_rmsnorm(x, eps=0.0)
