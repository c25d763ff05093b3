"""The cache's descriptor as a C caller fills it: what a format does not use is not read."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_gpu_cache import _fill, _gen, _make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", [("bf16", torch.bfloat16), ("fp16", torch.float16)])
@pytest.mark.parametrize("T,G,have", [(1, 4, 1000), (40, 4, 20), (40, 4, 3000)])
def test_scales_of_a_16_bit_cache_are_not_read(T, G, have, fmt, dtype):
    lib, heads, D = qlin.load_library(), 2, 64
    c = _make([have], [T], heads, D, 16, fmt)
    _fill(c, [have], [T])
    q = torch.randn(T, heads * G, D, generator=_gen(5), device="cuda").to(dtype)
    want = qlin.qlin_cache_attention(c, q, 0.125)
    three = torch.full((1,), 3.0, device="cuda")
    cache = qlin.CacheDesc(c.k.data_ptr(), c.v.data_ptr(), *c.k.stride()[:3], *c.v.stride()[:3], c.page_table.data_ptr(),
                           c.page_table.stride(0), c.cached.data_ptr(), c.q_start.data_ptr(), three.data_ptr(),
                           three.data_ptr(), 1, c.k.shape[0], 16, c.page_table.shape[1], heads, D,
                           qlin._CACHE_FORMATS[c.k.dtype])
    out, ws = torch.empty_like(q), qlin.alloc_cache_attention_workspace()
    args = qlin.CacheAttentionDesc(q.data_ptr(), out.data_ptr(), None, None, *q.stride()[:2], *out.stride()[:2], 0, T, 0.125,
                                   heads * G, 0, qlin._FLOAT16[dtype])
    assert lib.qlin_cache_attention(ctypes.byref(cache), ctypes.byref(args), ws.data_ptr(), ws.numel(),
                                    torch.cuda.current_stream().cuda_stream) == 0
    assert qlin.qlin_sync_status() == 0
    assert torch.equal(out, want)
