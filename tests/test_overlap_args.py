"""Outputs that lie over an input in another arrangement, or over themselves, are refused
before any launch (no GPU needed)."""
import ctypes

import pytest

pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin

INVALID = 1
K = 256


@pytest.fixture(scope="module")
def lib():
    from paper_2609_21849_gb300 import build
    build.build()
    return qlin.load_library()


# addresses that are never dereferenced
def _norm(**kw):
    d = dict(x=16, residual=32, sum=48, weight=64, x_stride=K, residual_stride=K, sum_stride=K, M=4, K=K, eps=1e-6,
             dtype=1)
    d.update(kw)
    return ctypes.byref(qlin.RMSNormDesc(*[d[n] for n, _ in qlin.RMSNormDesc._fields_]))


@pytest.mark.parametrize("kw,y", [
    (dict(sum=16, sum_stride=2 * K), 80), (dict(sum=32, residual_stride=2 * K), 80),   # the sum over x, over residual
    (dict(x_stride=2 * K), 16), (dict(residual_stride=2 * K), 32), ({}, 48)])          # y over each, over the sum
def test_norm(lib, kw, y):
    assert lib.qlin_rmsnorm(_norm(**kw), y, None) == INVALID
    if y == 80:
        fp8 = ctypes.byref(qlin.FP8Desc(96, 112, 4, K, 1))
        assert lib.qlin_rmsnorm_fp8(_norm(**kw), None, fp8, None) == INVALID
        fp4 = ctypes.byref(qlin.NVFP4Desc(96, 112, 128, 4, K))
        assert lib.qlin_rmsnorm_nvfp4(_norm(**kw), 144, fp4, None) == INVALID


def test_residual_of_a_linear(lib):
    e = ctypes.byref(qlin.EpilogueDesc(None, 48, 2 * K, 0))   # over y, rows further apart than y's
    assert lib.qlin_linear_bf16(16, 128, 32, 4, K, 128, e, 48, None) == INVALID
    r = ctypes.byref
    a8, w8 = qlin.FP8Desc(16, 16, 4, 128, 1), qlin.FP8Desc(16, 16, K, 128, 1)
    assert lib.qlin_linear_fp8(r(a8), r(w8), e, 48, None, None, 0, None) == INVALID
    a4, w4 = qlin.NVFP4Desc(16, 16, 16, 4, 128), qlin.NVFP4Desc(16, 16, 16, K, 128)
    assert lib.qlin_linear_nvfp4(r(a4), r(w4), e, 48, None, None, 0, None) == INVALID


@pytest.mark.parametrize("kw", [dict(y_head_stride=0), dict(y_token_stride=0), dict(y_head_stride=64),
                                dict(y_head_stride=-64), dict(y_token_stride=127),
                                dict(y=16, x_head_stride=0, y_head_stride=0)])   # an expanded x in place
def test_rotated_heads_over_one_another(lib, kw):
    d = dict(x=16, y=32, x_token_stride=512, x_head_stride=128, y_token_stride=512, y_head_stride=128, tokens=2,
             heads=4, positions=16, position_token_stride=1, position_axis_stride=0, turns=16, magnitude=1.0,
             head_dim=128, rot_dim=64, position_bits=32, axes=1, axis_pairs=(ctypes.c_int32 * 4)(32, 0, 0, 0),
             layout=0, inverse=0, dtype=1)
    d.update(kw)
    assert lib.qlin_rope(ctypes.byref(qlin.RopeDesc(*[d[n] for n, _ in qlin.RopeDesc._fields_])), None) == INVALID
