"""Attention of whole prompts: causal runs of thousands of tokens, alone, ragged and behind a cache."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_cache import FORMATS, _attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", FORMATS)
@pytest.mark.parametrize("cached,new,heads,G,D,page", [([0], [4608], 1, 2, 128, 64), ([0], [2049], 2, 1, 192, 16),
                                                       ([0, 100, 3000, 0], [1500, 2047, 1, 129], 1, 3, 64, 32),
                                                       ([8191], [1024], 1, 4, 80, 256),
                                                       ([0, 7], [300, 1025], 1, 2, 64, 24)])
def test_prompts(cached, new, heads, G, D, page, fmt, dtype):
    _attend(cached, new, heads, G, D, page, fmt, dtype, tree=False)
