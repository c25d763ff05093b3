"""Refusals of the block-scaled FP8 and the paged-cache calls before any launch (no GPU
needed), and the block-scaled linear's tile rules at the sizes that their comments quote."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest

torch = pytest.importorskip("torch")

from conftest import ROOT
from paper_2609_21849_gb300 import qlin

INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = 1, 2, 3, 6
BF16, FP16 = 1, 2
A16, A2 = 1 << 16, 1 << 20   # addresses that are never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_2609_21849_gb300 import build
    build.build()
    return qlin.load_library()


def _struct(cls, base, kw):
    d = dict.fromkeys((n for n, _ in cls._fields_), 0) | base | kw
    return ctypes.byref(cls(*[(ctypes.c_int32 * 4)(*d[n]) if n == "axis_pairs" else d[n] for n, _ in cls._fields_]))


def _block(**kw):
    return _struct(qlin.FP8BlockDesc, dict(codes=A16, scales=A16, rows=256, K=512, block_rows=1), kw)


def _cache(**kw):
    return _struct(qlin.CacheDesc, dict(
        k=A16, v=A2, k_page_stride=8192, k_slot_stride=512, k_head_stride=128, v_page_stride=8192, v_slot_stride=512,
        v_head_stride=128, page_table=A16, table_stride=8, cached=A16, q_start=A16, sequences=4, pages=64, page_size=16,
        table_width=8, heads=4, head_dim=128, format=BF16), kw)


def _append(**kw):
    return _struct(qlin.CacheAppendDesc, dict(
        k=A16, v=A16, q=A16, q_out=A2, k_token_stride=512, k_head_stride=128, v_token_stride=512, v_head_stride=128,
        q_token_stride=512, q_head_stride=128, q_out_token_stride=512, q_out_head_stride=128, tokens=4, positions=A16,
        position_token_stride=1, turns=A16, magnitude=1.0, q_heads=4, rot_dim=128, position_bits=32, axes=1,
        axis_pairs=(64, 0, 0, 0), layout=qlin._LAYOUTS["interleaved"], dtype=BF16), kw)


def _attention(**kw):
    return _struct(qlin.CacheAttentionDesc, dict(
        q=A16, out=A2, q_token_stride=1024, q_head_stride=128, out_token_stride=1024, out_head_stride=128, tokens=4,
        scale=0.1, q_heads=8, dtype=BF16), kw)


def test_scales_of_a_block_operand(lib):
    assert lib.qlin_fp8_block_scales(1, 64, 1) == 1
    assert lib.qlin_fp8_block_scales(129, 320, 1) == 3 * 129
    assert lib.qlin_fp8_block_scales(129, 320, 128) == 3 * 2
    for bad in ((0, 64, 1), (1, 96, 1), (1, 0, 1), (1, 64, 2)):
        assert lib.qlin_fp8_block_scales(*bad) == 0


def test_quantizer_refusals(lib):
    call = lib.qlin_quantize_fp8_block
    assert call(None, BF16, 512, _block(), None) == INVALID
    assert call(A16, BF16, 512, None, None) == INVALID
    assert call(A16, 3, 512, _block(), None) == INVALID
    assert call(A16, BF16, 511, _block(), None) == INVALID
    assert call(A16, BF16, 516, _block(), None) == MISALIGNED
    assert call(A16 + 2, BF16, 512, _block(), None) == MISALIGNED
    for kw, status in ((dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(rows=0), INVALID),
                       (dict(K=96), INVALID), (dict(block_rows=64), INVALID), (dict(codes=A16 + 8), MISALIGNED),
                       (dict(scales=A16 + 2), MISALIGNED), (dict(rows=2**31), UNSUPPORTED)):
        assert call(A16, BF16, 512, _block(**kw), None) == status, kw


def test_block_linear_refusals(lib):
    call = lib.qlin_linear_fp8_block
    w = lambda **kw: _block(**(dict(block_rows=128) | kw))  # noqa: E731
    assert call(None, w(), None, A16, None) == INVALID
    assert call(_block(), None, None, A16, None) == INVALID
    assert call(_block(), w(), None, None, None) == INVALID
    assert call(_block(), w(), None, A16 + 8, None) == MISALIGNED
    assert call(_block(block_rows=128), w(), None, A16, None) == INVALID
    assert call(_block(), w(block_rows=1), None, A16, None) == INVALID
    assert call(_block(), w(K=256), None, A16, None) == INVALID
    assert call(_block(), w(rows=96), None, A16, None) == INVALID
    assert call(_block(rows=2**32), w(), None, A16, None) == UNSUPPORTED
    for kw, status in ((dict(act=9), INVALID), (dict(residual=A16, residual_stride=255), INVALID),
                       (dict(bias=A16 + 2), MISALIGNED), (dict(residual=A16 + 8, residual_stride=256), MISALIGNED),
                       (dict(residual=A16, residual_stride=260), MISALIGNED)):
        assert call(_block(), w(), _struct(qlin.EpilogueDesc, {}, kw), A16, None) == status, kw


CACHE = [(dict(k=None), INVALID), (dict(v=None), INVALID), (dict(page_table=None), INVALID),
         (dict(cached=None), INVALID), (dict(q_start=None), INVALID), (dict(sequences=0), INVALID),
         (dict(pages=0), INVALID), (dict(page_size=0), INVALID), (dict(table_width=0), INVALID),
         (dict(heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(format=0), INVALID), (dict(format=4), INVALID),
         (dict(format=3), INVALID), (dict(format=3, k_scale=A16), INVALID), (dict(k_page_stride=-8), INVALID),
         (dict(v_head_stride=-8), INVALID), (dict(table_stride=7), INVALID), (dict(head_dim=272), UNSUPPORTED),
         (dict(heads=65537), UNSUPPORTED), (dict(sequences=2**24 + 1), UNSUPPORTED),
         (dict(page_table=A16 + 2), MISALIGNED), (dict(cached=A16 + 1), MISALIGNED),
         (dict(format=3, k_scale=A16, v_scale=A16 + 2), MISALIGNED)]


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_refusals(lib, kw, status):
    assert lib.qlin_cache_append(_cache(**kw), _append(), None) == status
    assert lib.qlin_cache_attention(_cache(**kw), _attention(), A16, 1 << 30, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(tokens=0), INVALID), (dict(dtype=3), INVALID),
    (dict(q_out=None), INVALID), (dict(q_heads=0), INVALID), (dict(dtype=FP16), UNSUPPORTED),
    (dict(rot_dim=0), INVALID), (dict(rot_dim=63), INVALID), (dict(rot_dim=130), INVALID), (dict(axes=0), INVALID),
    (dict(axes=5), INVALID), (dict(layout=7), INVALID), (dict(position_bits=16), INVALID),
    (dict(positions=None, axes=2, axis_pairs=(32, 32, 0, 0)), INVALID), (dict(axis_pairs=(63, 0, 0, 0)), INVALID),
    (dict(axes=2, axis_pairs=(65, -1, 0, 0)), INVALID), (dict(turns=A16 + 4), MISALIGNED),
    (dict(positions=A16 + 2), MISALIGNED), (dict(q_out=A16, q_out_token_stride=640), INVALID),
    (dict(q_out_token_stride=0), INVALID), (dict(q_out_head_stride=-64), INVALID), (dict(q=A16 + 1), MISALIGNED),
    (dict(k=A16 + 1), MISALIGNED), (dict(tokens=2**29), UNSUPPORTED), (dict(q_heads=65537), UNSUPPORTED)])
def test_append_refusals(lib, kw, status):
    assert lib.qlin_cache_append(_cache(), _append(**kw), None) == status


def test_append_cache_refusals(lib):
    assert lib.qlin_cache_append(None, _append(), None) == INVALID
    assert lib.qlin_cache_append(_cache(), None, None) == INVALID
    # the new rows would lie over one another (a cache that is only read may repeat pages)
    for kw in (dict(k_page_stride=0), dict(v_slot_stride=64), dict(k_head_stride=0)):
        assert lib.qlin_cache_append(_cache(**kw), _append(), None) == INVALID, kw
    assert lib.qlin_cache_append(_cache(k=A16 + 1), _append(), None) == MISALIGNED


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(tokens=0), INVALID), (dict(q_heads=0), INVALID),
    (dict(q_heads=6), INVALID), (dict(dtype=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=1e-40), INVALID), (dict(scale=2.0**127), INVALID),
    (dict(mask=A16, mask_words=0), INVALID), (dict(mask=A16, mask_words=1, mask_stride=-1), INVALID),
    (dict(out=A16, out_token_stride=2048), INVALID), (dict(out_head_stride=64), INVALID),
    (dict(out_token_stride=0), INVALID), (dict(dtype=FP16), UNSUPPORTED), (dict(tokens=2**24 + 1), UNSUPPORTED),
    (dict(q_heads=65540), UNSUPPORTED), (dict(tokens=2**24, q_heads=260), UNSUPPORTED),
    (dict(q=A16 + 8), MISALIGNED), (dict(out=A2 + 2), MISALIGNED), (dict(q_token_stride=1028), MISALIGNED),
    (dict(out_head_stride=132), MISALIGNED), (dict(lse=A16 + 2), MISALIGNED),
    (dict(mask=A16 + 4, mask_words=1, mask_stride=1), MISALIGNED)])
def test_attention_refusals(lib, kw, status):
    assert lib.qlin_cache_attention(_cache(), _attention(**kw), A16, 1 << 30, None) == status


def test_attention_cache_and_workspace_refusals(lib):
    call, size = lib.qlin_cache_attention, qlin.qlin_cache_attention_workspace_size()
    assert call(None, _attention(), A16, size, None) == INVALID
    assert call(_cache(), None, A16, size, None) == INVALID
    for kw, status in ((dict(head_dim=120), UNSUPPORTED), (dict(k=A16 + 8), MISALIGNED),
                       (dict(k_slot_stride=516), MISALIGNED),
                       (dict(format=3, k_scale=A16, v_scale=A16, v_head_stride=136), MISALIGNED)):
        assert call(_cache(**kw), _attention(), A16, size, None) == status, kw
    assert call(_cache(), _attention(), None, size, None) == WORKSPACE
    assert call(_cache(), _attention(), A16, size - 1, None) == WORKSPACE
    assert call(_cache(), _attention(), A16 + 8, size, None) == MISALIGNED


def test_python_refuses_tensors_of_the_host():
    bf = torch.zeros(4, 8, 64, dtype=torch.bfloat16)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    cache = qlin.PagedCache(torch.zeros(2, 16, 8, 64, dtype=torch.bfloat16), torch.zeros(2, 16, 8, 64, dtype=torch.bfloat16),
                            ints(1, 2), ints(1), ints(2))
    with pytest.raises(ValueError, match="x"):
        qlin.qlin_quantize_fp8_block(torch.zeros(4, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="A"):
        A = qlin.FP8BlockTensor(torch.zeros(4, 64, dtype=torch.uint8), torch.ones(1, 4), 4, 64, 1)
        qlin.qlin_linear_fp8_block(A, A)
    with pytest.raises(ValueError, match="k"):
        qlin.qlin_cache_append(cache, bf, bf)
    with pytest.raises(ValueError, match="q"):
        qlin.qlin_cache_attention(cache, bf, 0.1)


def _on_gpu():
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    return z, i, qlin.PagedCache(z(2, 16, 2, 64), z(2, 16, 2, 64), i(3, 2), i(3), i(4))


@pytest.mark.gpu
def test_python_checks_a_cache():
    z, i, good = _on_gpu()
    q, k = z(4, 4, 64), z(4, 2, 64)
    bad = [("cache", dict(v=z(2, 16, 2, 32))), ("cache", dict(v=good.v.half())), ("cache", dict(k=good.k.float())),
           ("cache", dict(k=good.k.cpu())), ("cache", dict(k=z(2, 16, 64, 2).transpose(2, 3))),
           ("cached", dict(cached=i(3).long())), ("cached", dict(cached=i(3, 1))), ("q_start", dict(q_start=i(3))),
           ("q_start", dict(q_start=i(8)[::2])), ("page_table", dict(page_table=i(2, 2))),
           ("page_table", dict(page_table=i(2, 3).t())), ("page_table", dict(page_table=i(3, 2).cpu()))]
    for name, kw in bad:
        c = qlin.PagedCache(**(vars(good) | kw))
        with pytest.raises(ValueError, match=name):
            qlin.qlin_cache_append(c, k, k)
        with pytest.raises(ValueError, match=name):
            qlin.qlin_cache_attention(c, q, 0.1)
    fp8 = qlin.PagedCache(good.k.to(torch.float8_e4m3fn), good.v.to(torch.float8_e4m3fn), good.page_table, good.cached,
                          good.q_start)
    with pytest.raises(ValueError, match="k_scale"):
        qlin.qlin_cache_attention(fp8, q, 0.1)
    fp8.k_scale = fp8.v_scale = torch.ones(1)
    with pytest.raises(ValueError, match="k_scale"):
        qlin.qlin_cache_append(fp8, k, k)


@pytest.mark.gpu
def test_python_checks_the_other_arguments():
    z, i, c = _on_gpu()
    q, k, plan = z(4, 4, 64), z(4, 2, 64), qlin.rope_plan(64)
    for kw in (dict(mask=i(4, 1)), dict(mask=i(3, 1).long()), dict(lse=z(4, 4)), dict(out=z(4, 4, 32)),
               dict(out=z(4, 4, 64).half()), dict(workspace=torch.zeros(1 << 27, dtype=torch.uint8)),
               dict(lse=torch.zeros(4, 8, device="cuda")[:, ::2])):
        with pytest.raises(ValueError, match=next(iter(kw))):
            qlin.qlin_cache_attention(c, q, 0.1, **kw)
    for args, name in (((z(4, 2, 32), k), "k"), ((k, z(3, 2, 64)), "v"), ((k, k, None, i(4)), "positions"),
                       ((k, k, plan, i(3)), "positions"), ((k, k, plan, i(4).float()), "positions"),
                       ((k, k, plan, None, z(4, 4, 32)), "q"), ((k, k, plan, None, None, q), "q_out")):
        with pytest.raises(ValueError, match=name):
            qlin.qlin_cache_append(c, *args)
    for call in (lambda: qlin.qlin_cache_attention(c, q, 0.0),
                 lambda: qlin.qlin_cache_attention(c, q, 0.1, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
                 lambda: qlin.qlin_cache_attention(c, q.half(), 0.1),
                 lambda: qlin.qlin_cache_append(c, k.half(), k.half())):
        with pytest.raises(qlin.QlinError):
            call()
    A, W = qlin.alloc_fp8_block(4, 128, 1), qlin.alloc_fp8_block(64, 128, 128)
    for bad in (qlin.FP8BlockTensor(A.codes[:3], A.scales, 4, 128, 1), qlin.FP8BlockTensor(A.codes, A.scales[:, :3], 4, 128, 1),
                qlin.FP8BlockTensor(A.codes, A.scales.cpu(), 4, 128, 1),
                qlin.FP8BlockTensor(A.codes, A.scales.double(), 4, 128, 1)):
        with pytest.raises(ValueError, match="A"):
            qlin.qlin_linear_fp8_block(bad, W)
    with pytest.raises(ValueError, match="y"):
        qlin.qlin_linear_fp8_block(A, W, y=z(4, 128))
    with pytest.raises(ValueError, match="out"):
        qlin.qlin_quantize_fp8_block(z(4, 64), out=A)
    with pytest.raises(qlin.QlinError):
        qlin.qlin_linear_fp8_block(A, A)
    assert qlin.qlin_sync_status() == 0


RULES = r"""
#include <cstdio>
#include "qlin_tiles.h"
int main() {
  long long m, n, k;
  while (std::scanf("%lld %lld %lld", &m, &n, &k) == 3)
    std::printf("%d %d %d\n", (int)qlin::few_block_tokens(m, n, k, 152), qlin::choose_block_split(m, n, k, 152),
                (int)qlin::choose_block_tile(m, n, k, 152));
}
"""
SHARED, SINGLE, SPLIT = range(3)


def test_block_linear_rules(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "main.cpp").write_text(RULES)
    csrc = os.path.join(ROOT, "paper_2609_21849_gb300", "csrc")
    subprocess.run([cxx, "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I" + csrc,
                    str(tmp_path / "main.cpp"), "-o", str(tmp_path / "main")], check=True)
    cases = [((1, 64, 64), 1, None, None), ((16, 2**30, 2**28), 1, None, None), ((17, 4096, 1088), 1, None, None),
             ((24, 5120, 3072), 1, None, None), ((24, 5120, 12288), 0, 2, SPLIT), ((300, 512, 12288), 0, 8, SPLIT),
             ((600, 512, 12288), 0, 4, SPLIT), ((300, 2112, 3072), 0, 2, SPLIT), ((300, 2112, 2048), 0, 1, SINGLE),
             ((1333, 2112, 256), 0, 1, SINGLE), ((1333, 2112, 1088), 0, 1, SHARED), ((300, 12288, 1088), 0, 1, SINGLE),
             ((4608, 12288, 3072), 0, 1, SHARED), ((2**31, 2**31 - 64, 2**31 - 64), 0, 1, None)]
    text = "".join("%d %d %d\n" % c[0] for c in cases)
    out = subprocess.run([str(tmp_path / "main")], input=text, capture_output=True, text=True, check=True)
    for (size, *want), line in zip(cases, out.stdout.splitlines()):
        for w, got in zip(want, map(int, line.split())):
            assert w is None or w == got, (size, want, line)
