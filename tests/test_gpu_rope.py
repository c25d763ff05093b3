"""Rotary positions against the formula in 64 bits.

Tolerances: the angle is exact to 2^-31 turn (2^-28 radians), cos and sin to two last
places, each product and the sum round once: 2^-21 (|a| + |b|) times the magnitude,
then one rounding to 16 bits."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

pytestmark = pytest.mark.gpu

UNIT = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}
LEAST = {torch.bfloat16: 2.0**-134, torch.float16: 2.0**-25}


def _expected(x, positions, plan, inverse):
    """(rotated x in 64 bits, |a| + |b| of each element's pair); the angle from the
    plan's turns by integers."""
    T, H, D = x.shape
    R, half = plan.rot_dim, plan.rot_dim // 2
    turns = [int(v) for v in plan.turns.cpu().numpy().view(np.uint64)]
    axis = np.repeat(np.arange(len(plan.axis_pairs)), plan.axis_pairs)
    pos = positions.cpu().numpy().reshape(T, -1)
    frac = np.array([[((int(pos[t, axis[i]]) * turns[i]) % 2**64) / 2**64 for i in range(half)] for t in range(T)])
    ang = torch.from_numpy(frac * 2 * math.pi * (-1 if inverse else 1)).to(x.device)[:, None]
    c, s, m = torch.cos(ang), torch.sin(ang), plan.magnitude
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    i = torch.arange(half, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if plan.layout == "interleaved" else (i, i + half)
    a, b = x.double()[..., ia], x.double()[..., ib]
    y[..., ia], y[..., ib] = m * (a * c - b * s), m * (a * s + b * c)
    size[..., ia] = size[..., ib] = m * (a.abs() + b.abs())
    return y, size


def _check(y, x, positions, plan, inverse=False):
    want, size = _expected(x, positions, plan, inverse)
    u, low = UNIT[x.dtype], LEAST[x.dtype]
    off = (y.double() - want).abs() - (u * want.abs() + (1 + u) * 2.0**-21 * size + low)
    assert off.max() <= 0, off.max().item()
    assert torch.equal(y[..., plan.rot_dim:], x[..., plan.rot_dim:])


def _x(T, H, D, dtype, seed=0, wide=0, first=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(T, first + H * D + wide, generator=g, device="cuda").to(dtype)
    return v[:, first:first + H * D].view(T, H, D) if wide or first else v.view(T, H, D)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,D,R", [(1, 1, 64, 64), (3, 40, 128, 64), (130, 5, 96, 96), (17, 24, 128, 128),
                                     (5, 3, 256, 128), (9, 7, 80, 20), (4, 2, 66, 34), (2, 1, 2, 2), (2, 3, 1024, 1024),
                                     (700, 1, 64, 32), (40, 97, 64, 48)])
def test_shapes_and_layouts(T, H, D, R, layout, dtype):
    x = _x(T, H, D, dtype, T + D)
    pos = torch.randint(0, 100000, (T,), device="cuda")
    plan = qlin.rope_plan(R, layout=layout)
    for inverse in (False, True):
        _check(qlin.qlin_rope(x, pos, plan, inverse=inverse), x, pos, plan, inverse)
    assert qlin.qlin_sync_status() == 0


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_scalings_against_real_angles(scaling):
    # the angles here from 64-bit reals, not from the plan: position * f is right to
    # 2^20 * 2^-52 radians
    T, H, R = 64, 2, 64
    x = _x(T, H, R, torch.float16, 1)
    pos = torch.randint(0, 1 << 20, (T,), device="cuda", dtype=torch.int32)
    plan = qlin.rope_plan(R, layout="half", scaling=scaling, factor=16.0, trained_length=4096)
    i = np.arange(R // 2)
    f = 10000.0 ** (-2.0 * i / R)
    if scaling == "linear":
        f = f / 16
    elif scaling == "ntk":
        f = (10000.0 * 16 ** (R / (R - 2))) ** (-2.0 * i / R)
    elif scaling == "yarn":
        at = lambda n: R * math.log(4096 / (n * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
        lo, hi = math.floor(at(32)), math.ceil(at(1))
        ramp = np.clip((i - lo) / (hi - lo), 0, 1)
        f = f * (1 - ramp) + f / 16 * ramp
    m = 0.1 * math.log(16) + 1 if scaling == "yarn" else 1.0
    ang = (pos.double()[:, None] * torch.from_numpy(f).cuda())[:, None]
    a, b = x[..., :R // 2].double(), x[..., R // 2:].double()
    want = torch.cat([a * torch.cos(ang) - b * torch.sin(ang), a * torch.sin(ang) + b * torch.cos(ang)], 2) * m
    size = torch.cat([a.abs() + b.abs()] * 2, 2) * m
    y = qlin.qlin_rope(x, pos, plan)
    off = (y.double() - want).abs() - (2.0**-11 * want.abs() + 2.0**-20 * size + 2.0**-25)
    assert off.max() <= 0


def test_positions_beyond_32_bits_and_negative():
    pos = torch.tensor([0, 1, -1, -4097, 2**31 - 1, -2**31, 2**31, 2**40 + 12345, 2**62 + 1, -2**63],
                       dtype=torch.int64, device="cuda")
    x = _x(len(pos), 3, 128, torch.bfloat16, 2)
    for layout in ("half", "interleaved"):
        plan = qlin.rope_plan(128, layout=layout)
        _check(qlin.qlin_rope(x, pos, plan), x, pos, plan)
        p32 = pos[:6].to(torch.int32)
        _check(qlin.qlin_rope(x[:6], p32, plan), x[:6], p32, plan)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("sizes", [(16, 56, 56), (32, 32), (8, 8, 8, 8), (0 + 2, 62)])
def test_several_axes(sizes, layout):
    T, R = 33, sum(sizes)
    x = _x(T, 6, 128, torch.bfloat16, 3)
    wide = torch.randint(-50, 5000, (T, 7), device="cuda", dtype=torch.int32)
    plan = qlin.rope_plan(sizes, layout=layout)
    pos = wide[:, 1:1 + len(sizes)]                       # strided positions
    y = qlin.qlin_rope(x, pos, plan)
    _check(y, x, pos.contiguous(), plan)
    assert R <= 128
    flipped = wide.t().contiguous().t()[:, 1:1 + len(sizes)]   # the axes apart
    assert torch.equal(qlin.qlin_rope(x, flipped, plan), y)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("wide,first", [(64, 0), (8, 8), (3, 0), (7, 1), (1, 3)])
def test_strides_alignment_and_in_place(wide, first, layout):
    # rows whose length or start is no multiple of eight elements included
    T, H, D, R = 21, 5, 64, 48
    plan = qlin.rope_plan(R, layout=layout)
    pos = torch.arange(T, device="cuda", dtype=torch.int32) * 37
    x = _x(T, H, D, torch.bfloat16, 4, wide, first)
    y = qlin.qlin_rope(x, pos, plan)
    _check(y, x, pos, plan)
    swapped = x.transpose(0, 1).contiguous().transpose(0, 1)      # heads outermost
    assert torch.equal(qlin.qlin_rope(swapped, pos, plan), y)
    out = torch.full((T, H + 2, D), 3.0, dtype=x.dtype, device="cuda")
    qlin.qlin_rope(x, pos, plan, out[:, 1:1 + H])
    assert torch.equal(out[:, 1:1 + H], y) and (out[:, 0] == 3).all() and (out[:, -1] == 3).all()
    base = torch.as_strided(x, (T, first + H * D + wide), (x.stride(0), 1), x.storage_offset() - first)
    before = base.clone()
    qlin.qlin_rope(x, pos, plan, x)
    assert torch.equal(x, y)
    assert torch.equal(base[:, :first], before[:, :first]) and torch.equal(base[:, first + H * D:], before[:, first + H * D:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_inverse_is_the_gradient(layout):
    # The rotation is linear: its differences along the unit vectors are its columns.
    # A head per unit vector gives all of them; the inverse's are the transpose, to
    # the two roundings.
    D, R = 32, 24
    plan = qlin.rope_plan(R, layout=layout, scaling="yarn", factor=8.0)
    eye = torch.eye(D, device="cuda").view(1, D, D)
    x0 = torch.randn(1, D, D, device="cuda").half()
    for p in (1, 777, 123456):
        pos = torch.tensor([p], device="cuda")
        h = eye.half()
        cols = qlin.qlin_rope(h, pos, plan).double()[0]                  # row j: column j of the rotation
        back = qlin.qlin_rope(h, pos, plan, inverse=True).double()[0]
        assert (cols - back.t()).abs().max() <= 2 * 2.0**-11 * 1.3
        # against the formula: the gradient of sum(g * rope(x)) by the transpose
        g = x0.double()[0]
        want = g @ cols.t()
        got = qlin.qlin_rope(x0, pos, plan, inverse=True).double()[0]
        assert (got - want).abs().max() <= 2.0**-9 * (2 * g.abs().max().item() * 1.3)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,R", [(80, 40), (80, 20), (72, 72), (24, 12), (96, 24), (88, 4), (40, 36), (88, 88), (200, 88)])
def test_rotations_of_any_width_beside_elements_that_pass(D, R, layout):
    # whatever is past the rotation, NaN among it, stays bit for bit
    for T, H in ((70, 1), (33, 6)):
        x = _x(T, H, D, torch.bfloat16, D + R)
        x.view(torch.int16)[..., R:] = torch.randint(-2**15, 2**15, (T, H, D - R), device="cuda").to(torch.int16)
        pos = torch.randint(0, 5000, (T,), device="cuda")
        plan = qlin.rope_plan(R, layout=layout)
        y = qlin.qlin_rope(x, pos, plan)
        _check(y[..., :R].contiguous(), x[..., :R].contiguous(), pos, plan)
        assert torch.equal(y.view(torch.int16)[..., R:], x.view(torch.int16)[..., R:])
        place = x.clone()
        qlin.qlin_rope(place, pos, plan, place)
        assert torch.equal(place.view(torch.int16), y.view(torch.int16))
        odd = torch.zeros(T, H, D + 8, dtype=x.dtype, device="cuda")[..., :D].copy_(x)   # rows 16 bytes apart
        assert torch.equal(qlin.qlin_rope(odd, pos, plan).view(torch.int16), y.view(torch.int16))


def test_refusals_of_tensors():
    x = _x(4, 2, 64, torch.bfloat16)
    pos = torch.arange(4, device="cuda")
    plan = qlin.rope_plan(64)
    two = qlin.rope_plan((32, 32))
    for bad in (lambda: qlin.qlin_rope(x.float(), pos, plan), lambda: qlin.qlin_rope(x[0], pos, plan),
                lambda: qlin.qlin_rope(x.transpose(1, 2), pos, plan), lambda: qlin.qlin_rope(x, pos[:3], plan),
                lambda: qlin.qlin_rope(x, pos.float(), plan), lambda: qlin.qlin_rope(x, pos.cpu(), plan),
                lambda: qlin.qlin_rope(x, pos, two), lambda: qlin.qlin_rope(x, pos, plan, x[:3]),
                lambda: qlin.qlin_rope(x, pos, plan, x.half()), lambda: qlin.qlin_rope(x, pos, qlin.rope_plan(64, device="cpu"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(qlin.QlinError):
        qlin.qlin_rope(x, pos, qlin.rope_plan(66))
