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


@pytest.mark.parametrize("cache", ["bf16", "f16", "i8"])
@pytest.mark.parametrize("page", [16, 10])
@pytest.mark.parametrize("what", ["mask", "window_positions", "absent"])
def test_attend_weights_of_rows_left_out_beside_a_nan(dev, ref, cache, page, what):
    """A NaN in one attended row makes its head's weights NaN, but the weight of
    a row that is left out is not touched, bit for bit."""
    _case("attend nan weights", cache, page, what)
    rng = np.random.default_rng(page)
    lens = [300, 1200, 40]
    c = ref.Cache(rng, 3, -(-1200 // page), 2, page, 64, cache)
    use = np.zeros((3, 2, c.rows), bool)
    for b, n in enumerate(lens):
        use[b, :, :n] = True
    mask = position = q_pos = None
    window = 0
    if what == "mask":
        mask = (rng.random((3, c.rows)) < 0.6).astype(np.uint8)
        use &= mask[:, None] != 0
    elif what == "window_positions":
        window, q_pos = 500, np.full(3, c.rows, np.int32)
        position = rng.permuted(np.tile(np.arange(c.rows, dtype=np.int32), (3, 2, 1)), axis=-1)
        use &= position > c.rows - window
    else:
        for b, p in ((0, 1), (0, 4), (1, 0), (1, 37), (2, 1)):
            c.table[b, p] = -1 - p
            use[b, :, p * page:(p + 1) * page] = False
    for b in range(3):  # key-value head 1 of each sequence
        r = int(np.flatnonzero(use[b, 1])[-1])
        if cache == "i8":
            c.scale["k"][int(c.table[b, r // page]), 1, r % page] = np.nan
        else:
            c.view("k")[int(c.table[b, r // page]), 1, r % page, 5] = float("nan")
    q = rng.standard_normal((3, 8, 64)).astype(np.float32)
    start = rng.random((3, 2, c.rows)).astype(np.float32)
    a = Attend(dev, ref, c, q, "f32", lens, window, mask, position, q_pos, start)
    got = a.run()
    w = a.dw.cpu().numpy()
    assert np.array_equal(w[~use], start[~use])
    assert np.all(np.isnan(w[:, 1][use[:, 1]])) and np.all(np.isnan(got[:, 4:]))
    want, p = ref.attend64(c, a.q, lens, a.scale, window, mask, position, q_pos)
    assert _rel(got[:, :4], want[:, :4]) <= TOL["f32"]
    # (the sums of weights in fp32: a unit of 1 from each rounding)
    assert np.max(np.abs(w[:, 0] - start[:, 0] - p[:, 0])) <= 2e-6


def test_attend_weights_of_scores_past_the_range(dev, ref):
    """Attended scores of -infinity: weight 0 beside finite ones, and none at all
    where there are no others; NaN beside a NaN."""
    rng = np.random.default_rng(32)
    lens = [700, 700, 700]
    c = ref.Cache(rng, 3, 44, 1, 16, 64, "bf16")
    c.view("k")[:] = c.view("k").abs() + 0.5
    for b, r in ((0, 333), (2, 40)):
        c.view("k")[int(c.table[b, r // 16]), 0, r % 16] = 0  # score 0
    c.view("k")[int(c.table[2, 20]), 0, 3, 7] = float("nan")
    q = -(np.abs(rng.standard_normal((3, 4, 64))) + 0.5).astype(np.float32)
    a = Attend(dev, ref, c, q, "f32", lens, scale=1e37, weight=np.zeros((3, 1, c.rows), np.float32))
    got = a.run()
    w = a.dw.cpu().numpy()[:, 0, :700]
    one = np.zeros(700, np.float32)
    one[333] = 4
    assert np.array_equal(w[0], one) and np.array_equal(w[1], 0 * one) and np.all(np.isnan(w[2]))
    v = c.rows64("v", 0, 0, 700)[333]
    assert _rel(got[0], np.tile(v, (4, 1))) <= TOL["f32"] and np.all(got[1] == 0) and np.all(np.isnan(got[2]))


@pytest.mark.parametrize("cache", ["bf16", "f16", "i8"])
@pytest.mark.parametrize("power", [24, 25, 26, 27, 28, 60])
@pytest.mark.parametrize("sign", [1, -1])
def test_attend_large_scores(dev, ref, cache, power, sign):
    """Largest scores of +-2^power and up to twice that, in units of ln 2, in rows
    of equal keys: the softmax is even over these, exactly, so a head's weights sum
    to 1 and its outputs are the rows' mean."""
    _case("attend large scores", cache, power, sign)
    rng = np.random.default_rng(power)
    lens = [900, 90, 33]
    c = ref.Cache(rng, 3, 57, 2, 16, 64, cache)
    c.view("k")[:] = 0
    other = 0.5 if sign > 0 else 2.0  # of the top rows' score
    if cache == "i8":
        c.view("k")[..., 0] = 64
        c.scale["k"][:] = other / 64
    else:
        c.view("k")[..., 0] = other
    for b, n in enumerate(lens):
        for h in range(2):
            for r in rng.choice(n, 7, replace=False):
                page = int(c.table[b, r // 16])
                if cache == "i8":
                    c.scale["k"][page, h, r % 16] = 1 / 64
                else:
                    c.view("k")[page, h, r % 16, 0] = 1
    q = np.zeros((3, 16, 64), np.float32)
    q[..., 0] = sign * 2.0 ** power * (1 + rng.random((3, 16))) * np.log(2)
    a = Attend(dev, ref, c, q, "f32", lens, scale=1.0, weight=np.zeros((3, 2, c.rows), np.float32))
    got = a.run()
    want, p = ref.attend64(c, a.q, lens, 1.0)
    assert np.all(np.isfinite(got)) and _rel(got, want) <= TOL["f32"]
    assert _rel(a.dw.double().cpu().numpy(), p) <= TOL["f32"]
    assert np.allclose(p.sum(-1), 8)  # (of the reference: 8 heads a group)
    plain = Attend(dev, ref, c, q, "f32", lens, scale=1.0).run()
    assert np.all(np.isfinite(plain)) and _rel(plain, want) <= TOL["f32"]


@pytest.mark.parametrize("low,high", [(-37, -32), (30, 34)])
def test_attend_int8_scales_near_the_ends(dev, ref, low, high):
    """V scales near the least and the largest normal numbers."""
    rng = np.random.default_rng(37)
    lens = [700, 90, 33]
    c = ref.Cache(rng, 3, 44, 2, 16, 64, "i8")
    c.scale["v"] = (10.0 ** rng.uniform(low, high, c.scale["v"].shape)).astype(np.float32)
    Attend(dev, ref, c, rng.standard_normal((3, 8, 64)).astype(np.float32), "f32", lens).check(ref)


def test_cache_of_65535_sequences(dev, ref):
    """The most sequences that a cache may have: all of them appended to, attended to
    and cut down."""
    import paper_2601_07892_amd as sh
    rng = np.random.default_rng(33)
    batch, dim = 65535, 16
    c = ref.Cache(rng, batch, 1, 1, 8, dim, "f16")
    lens = rng.integers(0, 8, batch)
    q = rng.standard_normal((batch, 1, dim)).astype(np.float32)
    x = torch.from_numpy(rng.standard_normal((batch, 1, dim)).astype(np.float32)).to(dev)
    a = Attend(dev, ref, c, q, "f32", lens + 1, weight=np.zeros((batch, 1, 8), np.float32))
    d = sh.sherry_append_desc()
    seq = torch.arange(batch, dtype=torch.int32, device=dev)
    slot = torch.from_numpy(lens.astype(np.int32)).to(dev)
    d.k = d.v = x.data_ptr()
    d.seq, d.slot, d.pos, d.tokens = seq.data_ptr(), slot.data_ptr(), slot.data_ptr(), batch
    sh.sherry_cache_append(a.cd, d)
    torch.cuda.synchronize()
    page = torch.from_numpy(c.table[:, 0]).long()
    for name in "kv":
        c.view(name)[page, 0, torch.from_numpy(lens)] = x[:, 0].cpu().half()
        assert torch.equal(c.d[name].cpu(), c.pool[name])
    for w in (True, False):
        if not w:
            a = Attend(dev, ref, c, q, "f32", lens + 1)
        got = a.run()
        k, v = (c.view(n)[page, 0].double().numpy() for n in "kv")
        s = np.einsum("bd,brd->br", a.q[:, 0].astype(np.float64), k) * a.scale
        s[np.arange(8) > lens[:, None]] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        assert _rel(got[:, 0], np.einsum("br,brd->bd", p, v)) <= TOL["f32"]
        if w:
            assert _rel(a.dw.double().cpu().numpy()[:, 0], p) <= TOL["f32"]
    _evict(dev, ref, rng, "f16", list(lens + 1), 3, 1, dim, 8, recent=1)


@pytest.mark.parametrize("rows", [4000, 15000, 65000, 70000])
@pytest.mark.parametrize("cache", ["bf16", "i8"])
def test_evict_in_tables_far_wider_than_the_sequences(dev, ref, rows, cache):
    """Short sequences in every form that the table's width chooses."""
    _case("evict wide", rows, cache)
    lens = [300, 1, 0, 65, 2100, 64]
    _evict(dev, ref, np.random.default_rng(rows), cache, lens, 60, 2, 32, 16, recent=9, spare=(rows - 2100) // 16)


@pytest.mark.parametrize("weights", ["random", "rising", "few"])
def test_evict_sequences_past_65536_rows(dev, ref, weights):
    """Keys that no registers hold: random weights, every kept row moved in several
    lists, and weights of few values."""
    _case("evict long", weights)
    rng = np.random.default_rng(35)
    make = {"random": None, "few": lambda s: rng.integers(0, 3, s).astype(np.float32),
            "rising": lambda s: np.broadcast_to(np.arange(s[-1], dtype=np.float32), s).copy()}[weights]
    _evict(dev, ref, rng, "bf16", [90000, 70001], 34000, 1, 8, 64, make, recent=0 if weights == "rising" else 500)


@pytest.mark.parametrize("kind,cache,page", [("f32", "bf16", 16), ("bf16", "f16", 64), ("f32", "i8", 12)])
@pytest.mark.parametrize("weights", [False, True])
def test_attend_in_tables_far_wider_than_the_sequences(dev, ref, kind, cache, page, weights):
    _case("attend wide", kind, cache, page, weights)
    rng = np.random.default_rng(36)
    lens = [300, 1, 0, 65, 2100, 64]
    c = ref.Cache(rng, 6, 40000 // page, 2, page, 64, cache)
    q = rng.standard_normal((6, 8, 64)).astype(np.float32)
    w = np.zeros((6, 2, c.rows), np.float32) if weights else None
    Attend(dev, ref, c, q, kind, lens, weight=w).check(ref)


@pytest.mark.parametrize("window", [1, 70, 2 ** 31 - 1])
def test_attend_windows_at_the_ends_of_32_bits(dev, ref, window):
    """Positions and windows whose difference does not fit 32 bits."""
    _case("attend window ends", window)
    rng = np.random.default_rng(38)
    lens = [100, 100, 40, 100, 33]
    c = ref.Cache(rng, 5, 7, 2, 16, 64, "bf16")
    position = rng.integers(-2 ** 31 + 1, 2 ** 31, (5, 2, c.rows)).astype(np.int32)
    position[:, :, ::3] = rng.integers(-200, 200, position[:, :, ::3].shape)
    position[3, :, ::5] = 2 ** 31 - 1
    q_pos = np.array([-5, -2 ** 31, -1, 2 ** 31 - 1, 60], np.int32)
    q = rng.standard_normal((5, 4, 64)).astype(np.float32)
    w = np.zeros((5, 2, c.rows), np.float32)
    Attend(dev, ref, c, q, "f32", lens, window, position=position, q_pos=q_pos, weight=w).check(ref)
