"""GPU tests of the e4m3 cache where its calls are easily wrong."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_cache_f8 import Attend, _case, dev, ref  # noqa: E402, F401


# ---- tokens past the table ---------------------------------------------------------

@pytest.mark.parametrize("kind,heads,kv,dim,length,new,window", [
    ("f32", 4, 1, 64, [4096], [500], 0), ("bf16", 4, 1, 128, [3900, 7], [700, 3], 0), ("f16", 6, 2, 64, [4000], [520], 2500),
    ("f32", 2, 2, 256, [100, 4096], [1, 300], 0)], ids=str)
def test_tokens_far_past_a_long_table(dev, ref, kind, heads, kv, dim, length, new, window):
    """Tiles of tokens behind the table's end, cut over workgroups: their costs count rows
    that the table does not have."""
    _case("tokens far past", kind, heads, kv, dim, length, new, window)
    c = ref.Cache(np.random.default_rng(30), len(length), 128, kv, 32, dim, [4096] * len(length))
    Attend(dev, ref, c, kind, heads, length, new, window=window).check(ref)
