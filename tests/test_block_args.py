"""Host side of the norm, the linears with an epilogue and the rotary positions (no
GPU needed): refusals before any launch, and the rotary frequencies."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

INVALID, UNSUPPORTED, MISALIGNED = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2609_21849_gb300 import build
    build.build()
    return qlin.load_library()


# addresses that are never dereferenced
def _norm(**kw):
    d = dict(x=16, residual=16, sum=16, weight=16, x_stride=256, residual_stride=256, sum_stride=256,
             M=4, K=256, eps=1e-6, dtype=1)
    d.update(kw)
    return ctypes.byref(qlin.RMSNormDesc(*[d[n] for n, _ in qlin.RMSNormDesc._fields_]))


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(M=0), INVALID), (dict(K=0), INVALID), (dict(K=96), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=math.inf), INVALID),
    (dict(eps=math.nan), INVALID), (dict(dtype=0), INVALID), (dict(dtype=3), INVALID),
    (dict(residual=None), INVALID),                      # a sum without a residual
    (dict(x_stride=255), INVALID), (dict(residual_stride=128), INVALID), (dict(sum_stride=0), INVALID),
    (dict(M=2**31), UNSUPPORTED), (dict(K=2**32, x_stride=2**32, residual_stride=2**32, sum_stride=2**32), UNSUPPORTED),
    (dict(x=24), MISALIGNED), (dict(residual=8), MISALIGNED), (dict(sum=2), MISALIGNED),
    (dict(weight=18), MISALIGNED), (dict(x_stride=260), MISALIGNED), (dict(residual_stride=257), MISALIGNED),
    (dict(sum_stride=258), MISALIGNED)])
def test_norm_refusals(lib, kw, status):
    assert lib.qlin_rmsnorm(_norm(**kw), 16, None) == status


def test_norm_output_refusals(lib):
    assert lib.qlin_rmsnorm(None, 16, None) == INVALID
    assert lib.qlin_rmsnorm(_norm(), None, None) == INVALID
    assert lib.qlin_rmsnorm(_norm(), 8, None) == MISALIGNED
    fp8 = lambda *a: ctypes.byref(qlin.FP8Desc(*a))  # noqa: E731
    assert lib.qlin_rmsnorm_fp8(_norm(), None, None, None) == INVALID
    # row scales with a static scale, a tensor scale without one
    assert lib.qlin_rmsnorm_fp8(_norm(), 16, fp8(16, 16, 4, 256, 1), None) == INVALID
    assert lib.qlin_rmsnorm_fp8(_norm(), None, fp8(16, 16, 4, 256, 0), None) == INVALID
    assert lib.qlin_rmsnorm_fp8(_norm(), None, fp8(16, 16, 5, 256, 1), None) == INVALID
    assert lib.qlin_rmsnorm_fp8(_norm(), None, fp8(24, 16, 4, 256, 1), None) == MISALIGNED
    assert lib.qlin_rmsnorm_fp8(_norm(), 18, fp8(16, 16, 4, 256, 0), None) == MISALIGNED
    fp4 = lambda *a: ctypes.byref(qlin.NVFP4Desc(*a))  # noqa: E731
    assert lib.qlin_rmsnorm_nvfp4(_norm(), None, fp4(16, 16, 16, 4, 256), None) == INVALID
    assert lib.qlin_rmsnorm_nvfp4(_norm(), 16, fp4(16, 16, 16, 4, 320), None) == INVALID
    assert lib.qlin_rmsnorm_nvfp4(_norm(), 18, fp4(16, 16, 16, 4, 256), None) == MISALIGNED


@pytest.mark.parametrize("ep,status", [
    ((16, None, 0, 5), INVALID), ((16, None, 0, -1), INVALID),   # no such activation
    ((None, 16, 255, 0), INVALID),                               # residual rows shorter than N
    ((18, None, 0, 0), MISALIGNED), ((None, 24, 256, 0), MISALIGNED), ((None, 16, 260, 0), MISALIGNED)])
def test_epilogue_refusals(lib, ep, status):
    e = ctypes.byref(qlin.EpilogueDesc(*ep))
    a4, w4 = qlin.NVFP4Desc(16, 16, 16, 4, 128), qlin.NVFP4Desc(16, 16, 16, 256, 128)
    a8, w8 = qlin.FP8Desc(16, 16, 4, 128, 1), qlin.FP8Desc(16, 16, 256, 128, 1)
    r = ctypes.byref
    assert lib.qlin_linear_nvfp4(r(a4), r(w4), e, 16, None, None, 0, None) == status
    assert lib.qlin_linear_fp8(r(a8), r(w8), e, 16, None, None, 0, None) == status
    assert lib.qlin_linear_bf16(16, 128, 16, 4, 256, 128, e, 16, None) == status
    assert lib.qlin_linear_fp16(16, 128, 16, 4, 256, 128, e, 16, None) == status


def test_linear_refusals(lib):
    r = ctypes.byref
    a4, w4 = qlin.NVFP4Desc(16, 16, 16, 4, 128), qlin.NVFP4Desc(16, 16, 16, 256, 128)
    assert lib.qlin_linear_nvfp4(None, r(w4), None, 16, None, None, 0, None) == INVALID
    assert lib.qlin_linear_nvfp4(r(a4), r(w4), None, None, None, None, 0, None) == INVALID   # nothing to write
    q4 = qlin.NVFP4Desc(16, 16, 16, 4, 128)
    assert lib.qlin_linear_nvfp4(r(a4), r(w4), None, 16, 16, r(q4), 192, None) == INVALID    # past N
    a8, w8 = qlin.FP8Desc(16, 16, 4, 128, 1), qlin.FP8Desc(16, 16, 256, 128, 1)
    assert lib.qlin_linear_fp8(r(a8), r(w8), None, None, None, None, 0, None) == INVALID
    q8 = qlin.FP8Desc(16, 16, 4, 256, 1)    # the re-quantized operand has one scale
    assert lib.qlin_linear_fp8(r(a8), r(w8), None, 16, 16, r(q8), 0, None) == INVALID
    w8 = qlin.FP8Desc(16, 16, 96, 128, 1)   # N % 64
    assert lib.qlin_linear_fp8(r(a8), r(w8), None, 16, None, None, 0, None) == INVALID
    # the plain GEMM still takes one scale for A only
    w8 = qlin.FP8Desc(16, 16, 256, 128, 1)
    assert lib.qlin_gemm_fp8(r(a8), r(w8), 16, None) == INVALID
    assert lib.qlin_linear_bf16(16, 96, 16, 4, 256, 96, None, 16, None) == INVALID
    assert lib.qlin_linear_fp16(16, 132, 16, 4, 256, 128, None, 16, None) == MISALIGNED


def _rope(**kw):
    d = dict(x=16, y=32, x_token_stride=512, x_head_stride=128, y_token_stride=512, y_head_stride=128,
             tokens=2, heads=4, positions=16, position_token_stride=1, position_axis_stride=0, turns=16,
             magnitude=1.0, head_dim=128, rot_dim=64, position_bits=32, axes=1,
             axis_pairs=(32, 0, 0, 0), layout=0, inverse=0, dtype=1)
    d.update(kw)
    d["axis_pairs"] = (ctypes.c_int32 * 4)(*d["axis_pairs"])
    return ctypes.byref(qlin.RopeDesc(*[d[n] for n, _ in qlin.RopeDesc._fields_]))


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(positions=None), INVALID), (dict(turns=None), INVALID),
    (dict(tokens=0), INVALID), (dict(heads=0), INVALID), (dict(rot_dim=0, axis_pairs=(0, 0, 0, 0)), INVALID),
    (dict(rot_dim=63), INVALID), (dict(rot_dim=130, axis_pairs=(65, 0, 0, 0)), INVALID),
    (dict(axes=0), INVALID), (dict(axes=5), INVALID), (dict(axis_pairs=(31, 0, 0, 0)), INVALID),
    (dict(axes=2, axis_pairs=(33, -1, 0, 0)), INVALID), (dict(position_bits=16), INVALID),
    (dict(layout=2), INVALID), (dict(dtype=3), INVALID),
    (dict(y=16, y_token_stride=1024), INVALID),          # in place with other strides
    (dict(head_dim=1088), UNSUPPORTED), (dict(tokens=2**31), UNSUPPORTED), (dict(heads=2**22), UNSUPPORTED),
    (dict(x=17), MISALIGNED), (dict(y=17), MISALIGNED), (dict(turns=12), MISALIGNED),
    (dict(positions=18), MISALIGNED), (dict(positions=20, position_bits=64), MISALIGNED)])
def test_rope_refusals(lib, kw, status):
    assert lib.qlin_rope(_rope(**kw), None) == status


def test_rope_frequencies():
    # turns are f / (2 pi) to 2^-51 of themselves: f carries the power's last-place
    # errors in 64 bits (2^-52 each side), the quotient one more; and to half a unit
    def check(turns, f):
        got = turns.numpy().view(np.uint64).astype(np.float64) * 2.0**-64
        want = np.array(f) / (2 * math.pi)
        assert np.all(np.abs(got - want) <= 2.0**-50 * want + 2.0**-65), (got, want)
    R, base, s = 64, 10000.0, 8.0
    f = [base ** (-2.0 * i / R) for i in range(R // 2)]
    t, m = qlin.qlin_rope_turns(R, base)
    check(t, f)
    assert m == 1.0 and t[0].item() == int(math.ldexp(1.0 / (2 * math.pi), 64))
    check(qlin.qlin_rope_turns(R, base, "linear", s)[0], [v / s for v in f])
    check(qlin.qlin_rope_turns(R, base, "ntk", s)[0],
          [(base * s ** (R / (R - 2))) ** (-2.0 * i / R) for i in range(R // 2)])
    check(qlin.qlin_rope_turns(2, base, "ntk", s)[0], [1 / s])
    # the blend: pairs that turn more than 32 times over 4096 positions keep f, those
    # that turn less than once take f / s, and the rest falls between, in order
    t, m = qlin.qlin_rope_turns(R, base, "yarn", s, 4096)
    got = t.numpy().view(np.uint64).astype(np.float64) * 2.0**-64 * 2 * math.pi
    turns_over = np.array(f) * 4096 / (2 * math.pi)
    ratio = got / np.array(f)
    assert np.allclose(ratio[turns_over > 40], 1.0, rtol=1e-12)
    assert np.allclose(ratio[turns_over < 0.8], 1 / s, rtol=1e-12)
    assert np.all(np.diff(ratio) <= 1e-15) and abs(m - (0.1 * math.log(s) + 1)) < 1e-7


@pytest.mark.parametrize("args", [(63,), (0,), (64, 1.0), (64, math.inf), (64, 1e4, "linear", 0.5),
                                  (64, 1e4, "ntk", math.nan), (64, 1e4, "yarn", 2.0, 0.0),
                                  (64, 1e4, "yarn", 2.0, 4096, 1.0, 1.0), (64, 1e4, "yarn", 2.0, 4096, 32, 0.0)])
def test_rope_frequency_refusals(args):
    with pytest.raises(qlin.QlinError) as e:
        qlin.qlin_rope_turns(*args)
    assert e.value.status == INVALID


def test_python_names_are_checked():
    with pytest.raises(ValueError):
        qlin.qlin_rope_turns(64, scaling="cubic")
    with pytest.raises(ValueError):
        qlin.rope_plan(64, layout="thirds", device="cpu")
    with pytest.raises(ValueError):
        qlin.rope_plan((16,) * 5, device="cpu")
    p = qlin.rope_plan((16, 56, 56), layout="interleaved", device="cpu")
    assert p.rot_dim == 128 and p.axis_pairs == (8, 28, 28)
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for call in (lambda: qlin.qlin_rmsnorm(x), lambda: qlin.qlin_linear_bf16(x, x),
                 lambda: qlin.qlin_rope(x.view(4, 1, 64), torch.zeros(4, dtype=torch.int32), p)):
        with pytest.raises(ValueError, match="CUDA"):   # no tensors of the host
            call()
