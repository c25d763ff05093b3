"""One key far above very many others: what these weigh together stays in the output.

The kernels hold P in 16 bits with the row's maximum at 2^15 (few rows) or at 2^7 and more (many) where
the type is fp16, whose steps below its normals are 2^-24: relative to the largest weight a weight w
is off by 2^-11 w or 2^-40 (few) or 2^-32 (many).  bf16 has the exponents of fp32, so there it is 2^-8 w.
The rest as in the other tests of the attention: 2^-21 of an exponential and 2^-22 of a score of at
most 28 ln 2 (products of one element, no sum), sums in steps of 16 keys at 2^-23 each."""
import math

import pytest

torch = pytest.importorskip("torch")

from paper_2609_21849_gb300 import qlin
from test_gpu_cache import FORMATS, LEAST, UNIT, _gen, _make, _slots

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("T,G", [(1, 4), (40, 4)])
@pytest.mark.parametrize("heads,have", [(1, 1 << 18), (320, 4096)])   # split among all CTAs, and whole in one
@pytest.mark.parametrize("where", [0.0, 0.4, 1.0])
def test_many_small_weights_beside_a_large_one(where, heads, have, T, G, fmt, dtype):
    D = 64
    c = _make([have], [T], heads, D, 64, fmt, junk=0.0)
    if fmt == "e4m3":
        c.k_scale.fill_(1.0)
        c.v_scale.fill_(1.0)
    at, g = _slots(c, 0, have + T), _gen(1)
    k = torch.zeros(have + T, 1, D, device="cuda")
    k[:, 0, 0] = torch.rand(have + T, generator=g, device="cuda") - 0.5
    top = int(where * (have - 1))
    k[top, 0, 0] = 28.0
    v = torch.rand(have + T, 1, D, generator=g, device="cuda") + 0.5
    v[top] = 0.0
    c.k[at], c.v[at] = (t.expand(-1, heads, -1).to(c.k.dtype) for t in (k, v))
    q = torch.zeros(T, heads * G, D, device="cuda", dtype=dtype)
    q[..., 0] = 1.0
    lse = torch.empty(T, heads * G, device="cuda")
    out = qlin.qlin_cache_attention(c, q, math.log(2), lse=lse)
    assert qlin.qlin_sync_status() == 0
    # every row sees the cache, and the new tokens up to its own
    s = c.k[at].double()[:, 0, 0] * math.log(2)
    w, vv = torch.exp(s - s[top]), c.v[at].double()[:, 0]
    want = torch.empty(T, D, dtype=torch.float64, device="cuda")
    total, size = torch.empty(T, dtype=torch.float64, device="cuda"), torch.empty_like(want)
    for t in range(T):
        n = have + t + 1
        total[t] = w[:n].sum()
        want[t], size[t] = w[:n] @ vv[:n] / total[t], vv[:n].sum(0) / total[t]
    u = 2.0**-8 if fmt == "bf16" else 2.0**-11
    floor = 0.0 if fmt == "bf16" else 2.0**-40 if T * G <= 16 else 2.0**-32
    L = have + T
    rel = 2 * (2.0**-21 + 2.0**-22 * 28 * math.log(2)) + (L / 16 + 64) * 2.0**-23
    tol = (u + rel) * want + floor * size
    off = (out.double() - want[:, None]).abs() - (tol + UNIT[dtype] * (want + tol) + LEAST[dtype])[:, None]
    assert off.max() <= 0, (off.max().item(), out.float().mean().item(), want.mean().item())
    want_lse = s[top] + torch.log(total)
    assert ((lse.double() - want_lse[:, None]).abs() <= rel + 2.0**-22 * want_lse[:, None].abs()).all()
