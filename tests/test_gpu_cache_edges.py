"""GPU parity of the paged cache at the ends of its ranges: how far a result of
16 bits is from its rounding, scores of any size, rows left out beside a NaN, many
sequences, and tables far wider than the sequences.  Helpers, references and the
2e-6 of fp32 results: test_gpu_cache.py."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_cache import TOL, Attend, _case, _evict, _rel, dev, ref  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("cache", ["bf16", "f16", "i8"])
def test_attend_16_bit_results_are_rounded_once(dev, ref, kind, cache):
    """With V all positive nothing cancels in sum p v / sum p, so each output's
    error before its rounding is the relative 2e-6 of an fp32 one, and no output
    is further from 64 bits than that and half a unit of its last place."""
    _case("attend rounding", kind, cache)
    rng = np.random.default_rng(31)
    lens = [700, 130, 1500, 33]
    c = ref.Cache(rng, 4, 94, 2, 16, 256, cache)
    for b in range(c.pages):
        c.view("v")[b] = c.view("v")[b].abs().clamp(min=1) if cache == "i8" else c.view("v")[b].abs() + 0.25
    q = rng.standard_normal((4, 16, 256)).astype(np.float32)
    weight = np.zeros((4, 2, c.rows), np.float32)
    for w in (None, weight):
        a = Attend(dev, ref, c, q, kind, lens, weight=w)
        got = a.run()
        want, p = ref.attend64(c, a.q, lens, a.scale)
        half = 2.0 ** (np.floor(np.log2(want)) - (8 if kind == "bf16" else 11))
        past = (np.abs(got - want) - half) / want
        assert past.max() <= TOL["f32"], (past.max(), (past > TOL["f32"]).sum())
    # the rows' weights come from the scores, which a q of 16 bits loses nothing of
    assert _rel(a.dw.double().cpu().numpy(), p) <= TOL["f32"]
