"""GPU parity of the paged key-value cache: append, attention of one new token
and eviction, against plain references (cache_reference.py).

Attention's tolerance, relative 2-norm of all outputs against 64 bits: fp32
outputs 2e-6 (operands of 22 bits and more, fp32 sums, an exponential within an
ulp of an argument below 2^5: together about 5 * 2^-22), bf16 and f16 outputs
the half ulp of their rounding (2^-9, 2^-12 relative to the binade's top, so at
most 2^-8, 2^-11 in a norm's terms) and as much again for 16-bit terms.
Accumulated weights: fp32 throughout, 2e-6, whatever the output's type (5e-5
with 16-bit inputs, whose scores keep 16 bits).  Append and eviction: bit for
bit."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOL = {"f32": 2e-6, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
WTOL = {"f32": 2e-6, "bf16": 5e-5, "f16": 5e-5}


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


@pytest.fixture(scope="module")
def ref():
    import cache_reference
    return cache_reference


def _case(*what):
    print("[case]", *what, file=sys.stderr, flush=True)


def _rel(x, y):
    n = np.linalg.norm(y)
    return np.linalg.norm(x - y) / (n if n else 1.0)


# ---- attention ------------------------------------------------------------------

class Attend:
    def __init__(self, dev, ref, c, q, kind, lens, window=0, mask=None, position=None, q_pos=None,
                 weight=None, scale=None, pad=0):
        import paper_2601_07892_amd as sh
        self.sh, self.c, self.lens, self.kind = sh, c, lens, kind
        self.batch, self.heads, self.dim = q.shape
        self.scale = float(np.float32(self.dim ** -0.5 if scale is None else scale))
        self.window, self.mask, self.position, self.q_pos = window, mask, position, q_pos
        self.cd = c.to(dev)
        row = self.heads * self.dim
        wide = torch.zeros((self.batch, row + pad), dtype=ref.TYPES[kind])
        wide[:, :row] = torch.from_numpy(q).reshape(self.batch, -1)
        self.q = wide[:, :row].float().numpy().reshape(q.shape)  # as rounded to its type
        self.qd = wide.to(dev)
        self.out = torch.full((self.batch, row + pad), float("nan"), dtype=ref.TYPES[kind], device=dev)
        up = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a, t)).to(dev)  # noqa: E731
        self.dl = up(lens, np.int32)
        self.dm, self.dp, self.dq = up(mask, np.uint8), up(position, np.int32), up(q_pos, np.int32)
        self.dw = up(weight, np.float32)
        d = self.d = sh.sherry_attend_desc()
        d.q, d.out, d.length = self.qd.data_ptr(), self.out.data_ptr(), self.dl.data_ptr()
        d.mask, d.position, d.q_pos = ref.at(self.dm), ref.at(self.dp), ref.at(self.dq)
        d.weight = ref.at(self.dw)
        d.q_stride = d.out_stride = row + pad
        d.mask_stride = mask.shape[-1] if mask is not None else 0
        d.row_stride = next((a.shape[-1] for a in (weight, position) if a is not None), 0)
        d.heads, d.type, d.window, d.scale = self.heads, ref.CODES[kind], window, self.scale
        n = sh.sherry_cache_attend_workspace(self.cd, d)
        assert n > 0
        self.ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=dev)  # (NaN everywhere)
        d.workspace, d.workspace_bytes = self.ws.data_ptr(), n

    def run(self):
        self.sh.sherry_cache_attend(self.cd, self.d)
        torch.cuda.synchronize()
        assert bool((self.ws[-64:] == 0xFF).all())  # nothing past the workspace
        row = self.heads * self.dim
        assert bool(torch.isnan(self.out[:, row:].float()).all())
        return self.out[:, :row].double().cpu().numpy().reshape(self.batch, self.heads, self.dim)

    def check(self, ref):
        before = None if self.dw is None else self.dw.double().cpu().numpy()
        got = self.run()
        want, p = ref.attend64(self.c, self.q, self.lens, self.scale, self.window, self.mask,
                               self.position, self.q_pos)
        assert np.all(np.isfinite(got))
        assert _rel(got, want) <= TOL[self.kind]
        for b in range(self.batch):  # a sequence's error does not hide behind the others'
            assert _rel(got[b], want[b]) <= 4 * TOL[self.kind], b
        empty = np.all(want == 0, axis=(1, 2))
        assert np.all(got[empty] == 0)
        if before is not None:
            w = self.dw.double().cpu().numpy()
            add = (w - before)[..., :p.shape[-1]]
            assert _rel(add, p) <= WTOL[self.kind]
            assert np.array_equal(w[..., p.shape[-1]:], before[..., p.shape[-1]:])
            assert np.array_equal(add[p == 0], np.zeros_like(add[p == 0]))


# q type, cache, heads, kv heads, head_dim, page size, lengths
SHAPES = [
    ("f32", "bf16", 8, 2, 64, 16, [1]),
    ("f32", "bf16", 8, 8, 128, 16, [31, 32, 33, 0, 1]),
    ("f32", "f16", 12, 4, 128, 64, [130, 15, 16, 17, 700]),
    ("f32", "i8", 32, 8, 128, 16, [1, 129, 500]),
    ("bf16", "bf16", 8, 2, 128, 32, [257, 64]),
    ("bf16", "f16", 6, 2, 64, 48, [100, 49, 1]),
    ("f16", "bf16", 4, 1, 256, 16, [65, 1000]),
    ("f16", "f16", 16, 1, 64, 128, [128, 129, 4000]),
    ("f16", "i8", 9, 3, 64, 16, [95, 96, 97]),
    ("bf16", "i8", 5, 1, 256, 32, [333, 2]),
    ("f32", "f16", 40, 2, 256, 16, [77, 160]),     # 20 query heads a group: two tiles of 16
    ("f32", "bf16", 33, 1, 64, 16, [200]),         # 33: three
    ("f32", "bf16", 4, 4, 80, 16, [50, 3]),        # head sizes between the padded ones
    ("f32", "f16", 4, 2, 8, 16, [50, 129]),
    ("f32", "bf16", 4, 2, 200, 32, [129, 40]),
    ("bf16", "i8", 4, 2, 112, 16, [129, 40]),
    ("f32", "bf16", 8, 2, 64, 1, [1, 40, 0]),      # pages that end anywhere in a tile
    ("f32", "bf16", 8, 2, 128, 7, [100, 350]),
    ("f16", "f16", 8, 2, 128, 20, [19, 20, 21, 333]),
    ("f32", "i8", 8, 2, 128, 12, [250, 1]),
    ("bf16", "bf16", 8, 2, 256, 100, [99, 1000]),
    ("f32", "i8", 4, 2, 48, 5, [77]),
]


@pytest.mark.parametrize("kind,cache,heads,kv,dim,page,lens", SHAPES)
@pytest.mark.parametrize("weights", [False, True])
def test_attend(dev, ref, kind, cache, heads, kv, dim, page, lens, weights):
    _case("attend", kind, cache, heads, kv, dim, page, lens, weights)
    rng = np.random.default_rng(heads * 1000 + dim + page)
    width = max(1, -(-max(lens) // page)) + 1
    c = ref.Cache(rng, len(lens), width, kv, page, dim, cache, lens, extra=32)
    q = (rng.standard_normal((len(lens), heads, dim)) * 3).astype(np.float32)
    w = np.zeros((len(lens), kv, c.rows + 5), np.float32) if weights else None
    Attend(dev, ref, c, q, kind, lens, weight=w, pad=8).check(ref)


@pytest.mark.parametrize("kind,cache,page", [("f32", "bf16", 16), ("f32", "f16", 64), ("bf16", "i8", 32),
                                             ("f32", "bf16", 10), ("f16", "i8", 9)])
@pytest.mark.parametrize("what", ["mask", "mask_all", "window", "window_positions", "both"])
def test_attend_left_out_rows(dev, ref, kind, cache, page, what):
    _case("attend rows", kind, cache, page, what)
    rng = np.random.default_rng(page)
    lens = [300, 1, 0, 64, 517]
    c = ref.Cache(rng, 5, -(-517 // page), 2, page, 128, cache, lens)
    q = (rng.standard_normal((5, 8, 128)) * 2).astype(np.float32)
    mask = position = q_pos = None
    window = 0
    if what in ("mask", "both"):
        mask = (rng.random((5, c.rows + 3)) < 0.7).astype(np.uint8) * 5
        mask[3] = 0  # nothing left
        mask[0, 64:128] = 0
    if what == "mask_all":
        mask = np.zeros((5, c.rows), np.uint8)
        mask[4, 516] = 1
    if what in ("window", "window_positions", "both"):
        window = 70
    if what in ("window_positions", "both"):
        position = rng.permuted(np.tile(np.arange(c.rows, dtype=np.int32), (5, 2, 1)), axis=-1)
        q_pos = np.array([c.rows, 0, 5, 200, 517], np.int32)
    if cache != "i8":  # rows that are left out hold anything
        pool = {n: c.view(n) for n in "kv"}
        for b, n in enumerate(lens):
            for r in range(n):
                if mask is not None and mask[b, r] == 0:
                    for name, x in (("k", float("nan")), ("v", float("inf"))):
                        pool[name][int(c.table[b, r // page]), :, r % page] = x
    weight = np.zeros((5, 2, c.rows), np.float32)
    Attend(dev, ref, c, q, kind, lens, window, mask, position, q_pos, weight).check(ref)


@pytest.mark.parametrize("window", [1, 31, 32, 33, 1000000])
def test_attend_window_edges(dev, ref, window):
    rng = np.random.default_rng(window)
    lens = [1, 31, 32, 33, 64, 400]
    c = ref.Cache(rng, 6, 25, 2, 16, 64, "bf16", lens)
    for b, n in enumerate(lens):  # rows before the window hold anything
        for r in range(max(0, n - window)):
            for name in "kv":
                c.view(name)[int(c.table[b, r // 16]), :, r % 16] = float("nan")
    q = rng.standard_normal((6, 4, 64)).astype(np.float32)
    Attend(dev, ref, c, q, "f32", lens, window).check(ref)


def test_attend_int8_scales_of_any_size(dev, ref):
    """V scales that rise and fall by powers of ten from row to row, zeros and
    negative ones among them; K scales that make some rows dominate."""
    rng = np.random.default_rng(14)
    lens = [700, 90, 33]
    c = ref.Cache(rng, 3, 44, 2, 16, 64, "i8")
    c.scale["v"] = (10.0 ** rng.uniform(-12, 12, c.scale["v"].shape)).astype(np.float32)
    c.scale["v"][rng.random(c.scale["v"].shape) < 0.1] = 0
    c.scale["v"][rng.random(c.scale["v"].shape) < 0.3] *= -1
    c.scale["k"][rng.random(c.scale["k"].shape) < 0.1] *= 10
    q = rng.standard_normal((3, 8, 64)).astype(np.float32)
    Attend(dev, ref, c, q, "f32", lens).check(ref)


@pytest.mark.parametrize("page", [16, 10])
@pytest.mark.parametrize("cache", ["bf16", "i8"])
def test_attend_absent_pages_and_wrong_lengths(dev, ref, page, cache):
    """Table entries out of range leave their rows out; lengths are clamped."""
    rng = np.random.default_rng(5)
    c = ref.Cache(rng, 4, 8, 2, page, 64, cache)
    c.table[0, 3] = -1
    c.table[1, :] = c.pages
    c.table[2, 0] = 2 ** 31 - 1
    lens = [8 * page, 5 * page, -7, 2 ** 31 - 1]
    q = rng.standard_normal((4, 4, 64)).astype(np.float32)
    Attend(dev, ref, c, q, "f32", lens).check(ref)


@pytest.mark.parametrize("cache", ["bf16", "f16"])
def test_attend_score_range(dev, ref, cache):
    """Large and tiny scores: one row takes all, or all rows the same; negative
    and zero scales; rows whose scores grow towards the end."""
    rng = np.random.default_rng(8)
    lens = [200, 200, 200]
    c = ref.Cache(rng, 3, 13, 1, 16, 64, cache, lens)
    q = rng.standard_normal((3, 4, 64)).astype(np.float32)
    q[0] *= 2.0 ** 60
    q[1] *= 2.0 ** -100
    q[2, 1] = 0
    for scale in (0.125, -0.5, 0.0):
        a = Attend(dev, ref, c, q, "f32", lens, scale=scale)
        got = a.run()
        want, _ = ref.attend64(c, a.q, lens, a.scale)
        # fp32 scores of 2^60 cannot order rows that 64 bits tell apart by
        # less than 2^-20: none of these are
        assert _rel(got, want) <= TOL["f32"], scale
    for r in range(200):
        c.view("k")[int(c.table[2, r // 16]), 0, r % 16] = r / 256
    q[2] = 1
    Attend(dev, ref, c, np.repeat(q[2:], 3, 0), "f32", lens, scale=0.125).check(ref)


def test_attend_values_that_are_not_finite(dev, ref):
    """A NaN or infinity in an attended row makes the outputs that it belongs to
    not finite, and no others."""
    rng = np.random.default_rng(9)
    lens = [100, 100, 100]
    c = ref.Cache(rng, 3, 7, 1, 16, 64, "bf16", lens)
    c.view("k")[int(c.table[0, 2]), 0, 3, 5] = float("nan")
    c.view("v")[int(c.table[1, 1]), 0, 2, 7] = float("inf")
    q = rng.standard_normal((3, 4, 64)).astype(np.float32)
    a = Attend(dev, ref, c, q, "f32", lens)
    got = a.run()
    assert np.all(np.isnan(got[0]))
    assert not np.any(np.isfinite(got[1, :, 7]))
    rest = np.delete(got[1], 7, axis=-1)
    assert np.all(np.isfinite(rest)) and np.all(np.isfinite(got[2]))


@pytest.mark.parametrize("lens", [[33, 1, 40], [1025, 2000, 4097]])
@pytest.mark.parametrize("cache", ["i8", "f16", "bf16"])
def test_attend_nan_alone_in_its_tile(dev, ref, cache, lens):
    """A NaN in the last row, which no other row shares a tile with."""
    rng = np.random.default_rng(16)
    c = ref.Cache(rng, 3, max(lens) // 16 + 1, 2, 16, 64, cache)
    for b in (0, 1):
        r = lens[b] - 1
        page = int(c.table[b, r // 16])
        if cache == "i8":
            c.scale["k"][page, 1, r % 16] = np.nan
        else:
            c.view("k")[page, 1, r % 16, 9] = float("nan")
    got = Attend(dev, ref, c, rng.standard_normal((3, 4, 64)).astype(np.float32), "f32", lens).run()
    assert np.all(np.isnan(got[:2, 2:]))
    assert np.all(np.isfinite(got[:2, :2])) and np.all(np.isfinite(got[2]))


@pytest.mark.parametrize("cache", ["i8", "f16", "bf16"])
def test_attend_q_of_any_size(dev, ref, cache):
    """Heads whose q are near the ends of fp32, or zero, with a scale that makes
    ordinary scores of them; a NaN or an infinity in q is its head's alone."""
    rng = np.random.default_rng(15)
    lens = [200, 33, 1]
    c = ref.Cache(rng, 3, 13, 2, 16, 128, cache)
    q = rng.standard_normal((3, 8, 128)).astype(np.float32)
    q[:, 3] = 0
    q[1, 2] /= 100
    top = np.float32(3.4e38 / np.abs(q).max())
    for by in (top, np.float32(2.0 ** 100), np.float32(2.0 ** -100)):
        Attend(dev, ref, c, q * by, "f32", lens, scale=0.0884 / float(by)).check(ref)
    q[0, 1, 17] = float("nan")
    q[1, 6, 127] = float("inf")
    q[2, 0, 0] = float("-inf")
    got = Attend(dev, ref, c, q, "f32", lens).run()
    for b, head in ((0, 1), (1, 6), (2, 0)):
        assert not np.any(np.isfinite(got[b, head]))
        assert np.all(np.isfinite(np.delete(got[b], head, axis=0)))


def test_attend_long_and_many(dev, ref):
    """A long sequence beside short ones (many splits of one), and more
    sequences than one wave counts."""
    rng = np.random.default_rng(10)
    lens = [20000, 3, 0, 700]
    c = ref.Cache(rng, 4, 1250, 1, 16, 64, "f16", None)
    q = rng.standard_normal((4, 4, 64)).astype(np.float32)
    Attend(dev, ref, c, q, "f32", lens, weight=np.zeros((4, 1, c.rows), np.float32)).check(ref)
    lens = list(rng.integers(0, 90, 150))
    lens[64:70] = [0] * 6
    c = ref.Cache(rng, 150, 6, 2, 16, 64, "bf16", None)
    q = rng.standard_normal((150, 4, 64)).astype(np.float32)
    Attend(dev, ref, c, q, "f32", lens, weight=np.zeros((150, 2, c.rows), np.float32)).check(ref)


@pytest.mark.parametrize("seed", range(24))
def test_attend_any_lengths(dev, ref, seed):
    """Random batches: which workgroups take which parts of which sequences
    follows from the lengths alone."""
    rng = np.random.default_rng(1000 + seed)
    batch, kv, group = int(rng.integers(1, 200)), int(rng.choice([1, 2, 3, 40])), int(rng.choice([1, 2, 5]))
    top = int(rng.choice([40, 600, 3000]) / (4 if kv == 40 else 1))
    lens = np.where(rng.random(batch) < 0.3, 0, np.exp(rng.random(batch) * np.log(top + 1)).astype(int))
    lens[rng.integers(0, batch)] = top
    page = int(rng.choice([16, 32, 11]))
    c = ref.Cache(rng, batch, -(-top // page), kv, page, int(rng.choice([16, 96, 144])),
                  str(rng.choice(["bf16", "f16", "i8"])))
    q = rng.standard_normal((batch, kv * group, c.dim)).astype(np.float32)
    _case("attend any", seed, batch, kv, group, top, page, c.dim, c.kind)
    weight = np.zeros((batch, kv, c.rows), np.float32) if seed % 3 == 0 else None
    Attend(dev, ref, c, q, "f32", lens, int(rng.choice([0, 0, 100])), weight=weight).check(ref)


def test_attend_offsets_past_32_bits(dev, ref):
    """Pools of more than 2^32 elements: the last pages (the rest is not set)."""
    import paper_2601_07892_amd as sh
    dim, page, kv = 128, 16, 2
    whole = page * kv * dim
    pages = (2 ** 32 + 2 ** 20) // whole
    k = torch.empty((pages, kv, page, dim), dtype=torch.float16, device=dev)
    v = torch.empty_like(k)
    rng = np.random.default_rng(11)
    small = ref.Cache(rng, 1, 4, kv, page, dim, "f16", [60])
    ids = torch.tensor([pages - 1, 3, pages - 2, pages // 2], device=dev)
    for name, pool in (("k", k), ("v", v)):
        pool[ids] = small.view(name)[torch.from_numpy(small.table[0]).long()].to(dev)
    q = rng.standard_normal((1, 4, dim)).astype(np.float32)
    a = Attend(dev, ref, small, q, "f32", [60])
    table = ids.to(torch.int32).view(1, 4).contiguous()
    a.cd.k, a.cd.v, a.cd.table, a.cd.pages = k.data_ptr(), v.data_ptr(), table.data_ptr(), pages
    a.check(ref)
    # and the append that fills them
    x = torch.from_numpy(rng.standard_normal((1, kv, dim)).astype(np.float32)).to(dev)
    i32 = lambda n: torch.tensor([n], dtype=torch.int32, device=dev)  # noqa: E731
    d = sh.sherry_append_desc()
    seq, slot = i32(0), i32(61)
    d.k = d.v = x.data_ptr()
    d.seq, d.slot, d.pos = seq.data_ptr(), slot.data_ptr(), slot.data_ptr()
    d.tokens = 1
    sh.sherry_cache_append(a.cd, d)
    torch.cuda.synchronize()
    assert torch.equal(k[pages // 2, :, 13], x[0].half()) and torch.equal(v[pages // 2, :, 13], x[0].half())


def test_attend_same_bits_every_time(dev, ref):
    rng = np.random.default_rng(12)
    lens = [900, 33, 410]
    c = ref.Cache(rng, 3, 60, 2, 16, 128, "bf16", lens)
    q = rng.standard_normal((3, 8, 128)).astype(np.float32)
    a = Attend(dev, ref, c, q, "f32", lens, weight=np.zeros((3, 2, c.rows), np.float32))
    first = a.run()
    w = a.dw.clone()
    for _ in range(3):
        a.dw.zero_()
        assert np.array_equal(a.run(), first) and torch.equal(a.dw, w)


# ---- append -----------------------------------------------------------------------

def _append(dev, ref, rng, kind, cache, tokens, heads, kv, dim, page, rot, pairs, pad=0, offset=0, inplace=False,
            with_q=True, marks=True):
    import paper_2601_07892_amd as sh
    batch, width = 3, 4
    c = ref.Cache(rng, batch, width, kv, page, dim, cache)
    rows = rng.permutation(batch * c.rows)[:tokens]
    seq, slot = (rows // c.rows).astype(np.int32), (rows % c.rows).astype(np.int32)
    pos = rng.integers(0, 50, tokens).astype(np.int32)
    bad = rng.choice(tokens, tokens // 4, replace=False)  # left out: every kind of it
    for n, i in enumerate(bad):
        what = n % 6
        if what == 0:
            seq[i] = -1
        elif what == 1:
            seq[i] = batch
        elif what == 2:
            slot[i] = -1
        elif what == 3:
            slot[i] = c.rows
        elif rot:
            pos[i] = 50 if what == 4 else -3
    t = ref.TYPES[kind]

    def rows_of(h):
        x = torch.from_numpy(rng.standard_normal((tokens, h * dim + pad)).astype(np.float32)).to(t)
        flat = torch.zeros(offset + x.numel(), dtype=t)
        flat[offset:] = x.reshape(-1)
        return flat, x[:, :h * dim].float().numpy().reshape(tokens, h, dim)

    (fq, q), (fk, k), (fv, v) = rows_of(heads), rows_of(kv), rows_of(kv)
    ang = rng.random((50, max(rot, 2) // 2)) * 6
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    cd = c.to(dev)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
    e = fq.element_size()
    dq, dk, dv = fq.to(dev), fk.to(dev), fv.to(dev)
    dout = dq if inplace else torch.full_like(dq, 7)
    hold = [up(x) for x in (seq, slot, pos, cos, sin)]
    w0 = rng.random((batch, kv, c.rows + 2)).astype(np.float32)
    p0 = rng.integers(0, 9, w0.shape).astype(np.int32)
    dw, dp = up(w0), up(p0)
    d = sh.sherry_append_desc()
    d.k, d.v = dk.data_ptr() + offset * e, dv.data_ptr() + offset * e
    if with_q:
        d.q, d.q_out = dq.data_ptr() + offset * e, dout.data_ptr() + offset * e
    d.seq, d.slot, d.pos = (x.data_ptr() for x in hold[:3])
    if rot:
        d.cos, d.sin = hold[3].data_ptr(), hold[4].data_ptr()
    if marks:
        d.weight, d.position, d.row_stride = dw.data_ptr(), dp.data_ptr(), c.rows + 2
    d.q_stride = d.q_out_stride = heads * dim + pad
    d.k_stride = d.v_stride = kv * dim + pad
    d.tokens, d.heads, d.type, d.rope_rows, d.rot_dim = tokens, heads, ref.CODES[kind], 50, rot
    d.pairing = sh.SHERRY_ROPE_PAIRS if pairs else sh.SHERRY_ROPE_HALVES
    sh.sherry_cache_append(cd, d)
    torch.cuda.synchronize()

    ok = (seq >= 0) & (seq < batch) & (slot >= 0) & (slot < c.rows)
    if rot:
        ok &= (pos >= 0) & (pos < 50)
        cs, sn = cos[np.clip(pos, 0, 49)], sin[np.clip(pos, 0, 49)]
        rq, rk = (ref.rotate32(x, cs, sn, rot, pairs) for x in (q, k))
    else:
        rq, rk = q, k
    want = fq.clone() if inplace else torch.full_like(fq, 7)
    if with_q:
        body = want[offset:].view(tokens, -1)
        rounded = torch.from_numpy(rq.reshape(tokens, -1)).to(t)
        for i in np.flatnonzero(ok):
            body[i, :heads * dim] = rounded[i]
    assert torch.equal(dout.cpu(), want)
    for name, x in (("k", rk), ("v", v)):
        full = c.pool[name].clone()
        pool = c.view(name, full)
        scale = None if c.scale[name] is None else c.scale[name].copy()
        for i in np.flatnonzero(ok):
            p, o = int(c.table[seq[i], slot[i] // page]), int(slot[i] % page)
            if cache == "i8":
                qq, s = ref.quantize32(x[i])
                pool[p, :, o] = torch.from_numpy(qq)
                scale[p, :, o] = s
            else:
                pool[p, :, o] = torch.from_numpy(x[i]).to(ref.TYPES[cache])
        assert torch.equal(c.d[name].cpu(), full), name
        if scale is not None:
            assert np.array_equal(c.ds[name].cpu().numpy(), scale), name
    if marks:
        for i in np.flatnonzero(ok):
            w0[seq[i], :, slot[i]] = 0
            p0[seq[i], :, slot[i]] = pos[i]
    assert np.array_equal(dw.cpu().numpy(), w0) and np.array_equal(dp.cpu().numpy(), p0)


@pytest.mark.parametrize("kind,cache,tokens,heads,kv,dim,page,rot,pairs,pad", [
    ("f32", "bf16", 1, 4, 1, 64, 16, 64, False, 0), ("f32", "i8", 40, 8, 2, 128, 16, 128, False, 0),
    ("bf16", "f16", 33, 4, 4, 256, 16, 128, False, 8), ("f16", "i8", 20, 6, 2, 80, 7, 80, False, 16),
    ("f32", "f16", 11, 3, 3, 8, 16, 6, False, 1), ("bf16", "bf16", 30, 4, 2, 64, 20, 64, True, 3),
    ("f32", "i8", 25, 2, 1, 48, 64, 20, True, 0), ("f32", "bf16", 17, 4, 2, 200, 5, 100, False, 4),
    ("f16", "f16", 9, 4, 2, 128, 16, 0, False, 0), ("f32", "bf16", 13, 4, 2, 72, 1, 34, False, 0)])
def test_append(dev, ref, kind, cache, tokens, heads, kv, dim, page, rot, pairs, pad):
    _case("append", kind, cache, tokens, heads, kv, dim, page, rot, pairs, pad)
    rng = np.random.default_rng(tokens)
    tokens = min(tokens, 12 * page)
    _append(dev, ref, rng, kind, cache, tokens, heads, kv, dim, page, rot, pairs, pad)


def test_append_alone_in_place_and_at_odd_addresses(dev, ref):
    rng = np.random.default_rng(3)
    _append(dev, ref, rng, "f32", "bf16", 20, 4, 2, 64, 16, 64, False, offset=1)
    _append(dev, ref, rng, "bf16", "i8", 20, 4, 2, 64, 16, 32, True, offset=3, with_q=False, marks=False)


def test_append_rotates_q_in_place(dev, ref):
    """q_out = q: the rotation's two halves of a row are read before either is
    written."""
    rng = np.random.default_rng(4)
    for dim, pairs, offset in ((64, False, 0), (128, False, 0), (256, False, 0), (256, True, 1), (72, False, 1)):
        _append(dev, ref, rng, "f32", "bf16", 40, 8, 2, dim, 16, dim, pairs, offset=offset, inplace=True)


def test_append_quantizes_edges(dev, ref):
    """Rows of zeros, of one value, and on rounding boundaries."""
    import paper_2601_07892_amd as sh
    rng = np.random.default_rng(6)
    c = ref.Cache(rng, 1, 1, 1, 16, 64, "i8")
    x = np.zeros((5, 1, 64), np.float32)
    x[1] = 3.5
    x[2] = (np.arange(64) - 31.5) * (127 / 63.5) / 2
    x[3] = rng.standard_normal(64) * 1e-38
    x[4, 0, 5] = -1e30
    cd = c.to(dev)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
    hold = [up(x), up(np.zeros(5, np.int32)), up(np.arange(5, dtype=np.int32))]
    d = sh.sherry_append_desc()
    d.k = d.v = hold[0].data_ptr()
    d.seq, d.slot, d.pos, d.tokens = hold[1].data_ptr(), hold[2].data_ptr(), hold[2].data_ptr(), 5
    sh.sherry_cache_append(cd, d)
    torch.cuda.synchronize()
    q, s = ref.quantize32(x)
    page = int(c.table[0, 0])
    got = c.view("k", c.d["k"].cpu())[page, 0, :5].numpy()
    assert np.array_equal(got, q[:, 0]) and np.array_equal(c.ds["v"].cpu().numpy()[page, 0, :5], s[:, 0])


# ---- eviction -----------------------------------------------------------------------

def _evict(dev, ref, rng, cache, lens, keep, kv, dim, page, weight=None, positions=True, recent=0, outs=True,
           spare=0):
    import paper_2601_07892_amd as sh
    batch = len(lens)
    width = max(1, -(-max(n for n in lens if n < 10 ** 6) // page)) + spare
    c = ref.Cache(rng, batch, width, kv, page, dim, cache, extra=16)
    shape = (batch, kv, c.rows + 3)
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32) if weight is None else weight(shape)
    pos = rng.permuted(np.tile(np.arange(shape[-1], dtype=np.int32) + 5, (batch, kv, 1)), axis=-1)
    frm = np.full(batch, shape[-1] + 5 - recent, np.int32) if recent is not None else None
    if not positions and frm is not None:
        frm = np.array([max(0, n - recent) for n in lens], np.int32)
    cd = c.to(dev)
    up = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a, t)).to(dev)  # noqa: E731
    dl, dw, dp, df = up(lens, np.int32), up(w, np.float32), up(pos, np.int32), up(frm, np.int32)
    oshape = (batch, kv, keep + 2)
    kept = torch.full(oshape, -9, dtype=torch.int32, device=dev)
    wo, po = torch.full(oshape, -9.0, device=dev), torch.full(oshape, -9, dtype=torch.int32, device=dev)
    lo = torch.full((batch,), -9, dtype=torch.int32, device=dev)
    d = sh.sherry_evict_desc()
    d.length, d.weight, d.position = dl.data_ptr(), dw.data_ptr(), dp.data_ptr() if positions else None
    d.recent_from, d.length_out, d.kept = ref.at(df), lo.data_ptr(), kept.data_ptr()
    if outs:
        d.weight_out, d.position_out = wo.data_ptr(), po.data_ptr()
    d.row_stride, d.out_stride, d.keep = shape[-1], keep + 2, keep

    want_k = np.full(oshape, -1, np.int32)
    want_w, want_p = np.zeros(oshape, np.float32), np.zeros(oshape, np.int32)
    pools = {n: c.pool[n].clone() for n in "kv"}
    scales = {n: None if c.scale[n] is None else c.scale[n].copy() for n in "kv"}
    for b in range(batch):
        n = max(0, min(lens[b], c.rows))
        for h in range(kv):
            ps = pos[b, h] if positions else np.arange(shape[-1])
            plan = ref.evict_plan(w[b, h], ps, None if frm is None else frm[b], n, keep)
            for i, src in enumerate(plan):
                want_k[b, h, i], want_w[b, h, i], want_p[b, h, i] = src, w[b, h, src], ps[src]
                if src != i:
                    (tp, to), (fp, fo) = ((int(c.table[b, x // page]), x % page) for x in (i, src))
                    for name in "kv":
                        c.view(name, pools[name])[tp, h, to] = c.view(name)[fp, h, fo]
                        if scales[name] is not None:
                            scales[name][tp, h, to] = c.scale[name][fp, h, fo]
    for a in (want_k, want_w, want_p):
        a[..., keep:] = -9
    for again in range(2):  # (a second call on the same lengths and weights changes nothing)
        sh.sherry_cache_evict(cd, d)
        torch.cuda.synchronize()
        assert np.array_equal(lo.cpu().numpy(), np.clip(lens, 0, min(keep, c.rows)))
        assert np.array_equal(kept.cpu().numpy(), want_k)
        if outs:
            assert np.array_equal(wo.cpu().numpy(), want_w, equal_nan=True)
            assert np.array_equal(po.cpu().numpy(), want_p)
        for name in "kv":
            assert torch.equal(c.d[name].cpu(), pools[name]), name
            if scales[name] is not None:
                assert np.array_equal(c.ds[name].cpu().numpy(), scales[name]), name


@pytest.mark.parametrize("cache,lens,keep,kv,dim,page,recent", [
    ("bf16", [100], 60, 2, 64, 16, 10), ("f16", [1, 0, 500, 64, 65], 64, 1, 128, 16, 5),
    ("i8", [300, 299, 10], 128, 2, 48, 7, 0), ("bf16", [1500, 1024, 1025], 1024, 1, 8, 64, 100),
    ("i8", [70, 3000], 1, 1, 256, 32, 0), ("f16", [40, 41], 500, 2, 64, 20, 3),
    ("bf16", [5000, 63, 4097], 2500, 1, 16, 128, 700), ("bf16", [200], 199, 3, 200, 16, None),
    ("f16", [40000], 20000, 1, 8, 256, 1000)])
def test_evict(dev, ref, cache, lens, keep, kv, dim, page, recent):
    _case("evict", cache, lens, keep, kv, dim, page, recent)
    _evict(dev, ref, np.random.default_rng(keep), cache, lens, keep, kv, dim, page, recent=recent)


@pytest.mark.parametrize("what", ["equal", "few", "zeros", "nan", "all_nan", "negative", "infinite", "rising",
                                  "falling", "all_recent"])
def test_evict_ties_and_values(dev, ref, what):
    rng = np.random.default_rng(2)

    def weight(shape):
        w = np.exp(rng.standard_normal(shape)).astype(np.float32)
        n = shape[-1]
        if what == "equal":
            w[:] = 0.25
        elif what == "few":
            w = rng.integers(0, 3, shape).astype(np.float32)
        elif what == "zeros":
            w[rng.random(shape) < 0.9] = 0
            w[rng.random(shape) < 0.3] *= -0.0
        elif what == "nan":
            w[rng.random(shape) < 0.5] = np.nan
            w[rng.random(shape) < 0.3] = -np.inf
        elif what == "all_nan":
            w[:] = np.nan
        elif what == "negative":
            w = rng.standard_normal(shape).astype(np.float32) * np.float32(1e-40)
        elif what == "infinite":
            w[rng.random(shape) < 0.5] = np.inf
        elif what == "rising":
            w[:] = np.arange(n)
        elif what == "falling":
            w[:] = -np.arange(n)
        return w

    for lens, keep in (([257, 90], 130), ([2100], 1000)):
        _evict(dev, ref, rng, "bf16", lens, keep, 2, 16, 16, weight, recent=9000 if what == "all_recent" else 7)


def test_evict_more_moves_than_are_matched_at_a_time(dev, ref):
    """Every kept row moves: the heaviest are the last ones, 20000 of 40000 (the
    matching list holds 16384)."""
    rng = np.random.default_rng(7)
    _evict(dev, ref, rng, "bf16", [40000], 20000, 1, 8, 64,
           lambda s: np.broadcast_to(np.arange(s[-1], dtype=np.float32), s).copy(), recent=0)


def test_evict_without_positions_or_copies(dev, ref):
    rng = np.random.default_rng(3)
    _evict(dev, ref, rng, "bf16", [200, 5], 100, 2, 64, 16, positions=False, recent=20)
    _evict(dev, ref, rng, "i8", [200, 5], 100, 2, 64, 16, outs=False, recent=20, spare=3)
    _evict(dev, ref, rng, "bf16", [200, -4, 10 ** 9], 100, 2, 64, 16)


def test_evict_absent_pages(dev, ref):
    """A row on a page out of range is not moved, nothing else is touched."""
    import paper_2601_07892_amd as sh
    rng = np.random.default_rng(13)
    c = ref.Cache(rng, 1, 8, 1, 16, 64, "bf16")
    c.table[0, 6] = c.pages
    c.table[0, 1] = -1
    cd = c.to(dev)
    w = torch.zeros((1, 1, 128), device=dev)
    w[..., 64:] = 1  # rows 64 .. 127 are kept and go to 0 .. 63
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32, device=dev)  # noqa: E731
    length, lo, kept = i32(1) + 128, i32(1), i32(1, 1, 64)
    d = sh.sherry_evict_desc()
    d.length, d.weight, d.length_out, d.kept = length.data_ptr(), w.data_ptr(), lo.data_ptr(), kept.data_ptr()
    d.row_stride, d.out_stride, d.keep = 128, 64, 64
    sh.sherry_cache_evict(cd, d)
    torch.cuda.synchronize()
    assert torch.equal(kept.cpu()[0, 0], torch.arange(64, 128, dtype=torch.int32))
    for name in "kv":
        want = c.pool[name].clone()
        pool = c.view(name, want)
        for i in range(64):
            if i // 16 == 1 or (i + 64) // 16 == 6:
                continue
            pool[int(c.table[0, i // 16]), 0, i % 16] = c.view(name)[int(c.table[0, (i + 64) // 16]), 0, i % 16]
        assert torch.equal(c.d[name].cpu(), want)


# ---- together -------------------------------------------------------------------------

def test_captured_step(dev, ref):
    """Append, attention with weights, eviction in a captured graph on another
    stream, replayed with other work between, against the same calls eagerly."""
    import paper_2601_07892_amd as sh
    rng = np.random.default_rng(21)
    lens = [100, 31, 250]
    c = ref.Cache(rng, 3, 17, 2, 16, 64, "bf16")
    q = rng.standard_normal((3, 8, 64)).astype(np.float32)
    a = Attend(dev, ref, c, q, "f32", [n + 1 for n in lens], weight=np.zeros((3, 2, c.rows), np.float32))
    up = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).to(dev)  # noqa: E731
    new = up(rng.standard_normal((3, 2, 64)), np.float32)
    seq, slot = up(np.arange(3), np.int32), up(lens, np.int32)
    ang = rng.random((300, 32))
    cos, sin = up(np.cos(ang), np.float32), up(np.sin(ang), np.float32)
    qin = torch.from_numpy(q).to(dev)
    ap = sh.sherry_append_desc()
    ap.q, ap.q_out, ap.k, ap.v = qin.data_ptr(), a.qd.data_ptr(), new.data_ptr(), new.data_ptr()
    ap.seq, ap.slot, ap.pos = seq.data_ptr(), slot.data_ptr(), slot.data_ptr()
    ap.cos, ap.sin, ap.weight, ap.row_stride = cos.data_ptr(), sin.data_ptr(), a.dw.data_ptr(), c.rows
    ap.tokens, ap.heads, ap.rope_rows, ap.rot_dim = 3, 8, 300, 64
    kept, wo = torch.zeros((3, 2, 64), dtype=torch.int32, device=dev), torch.zeros((3, 2, 64), device=dev)
    lo = torch.zeros(3, dtype=torch.int32, device=dev)
    ev = sh.sherry_evict_desc()
    ev.length, ev.weight, ev.length_out, ev.kept, ev.weight_out = (
        x.data_ptr() for x in (a.dl, a.dw, lo, kept, wo))
    ev.row_stride, ev.out_stride, ev.keep = c.rows, 64, 64
    start = {n: p.clone() for n, p in c.d.items()}

    def reset():
        for n in "kv":
            c.d[n].copy_(start[n])
        a.dw.zero_()
        a.out.zero_()
        kept.zero_()

    def step():
        sh.sherry_cache_append(a.cd, ap)
        sh.sherry_cache_attend(a.cd, a.d)
        sh.sherry_cache_evict(a.cd, ev)

    outs = lambda: [x.clone() for x in (a.out, a.dw, kept, wo, lo, c.d["k"], c.d["v"], a.qd)]  # noqa: E731
    reset()
    step()
    torch.cuda.synchronize()
    want = outs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(4):
        reset()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs(), want):
            assert torch.equal(x, y)
        junk = torch.randn(1 << 20, device=dev).sum().item()
        assert junk == junk
    with torch.cuda.stream(side):  # eagerly on a stream of its own
        reset()
        step()
    side.synchronize()
    for x, y in zip(outs(), want):
        assert torch.equal(x, y)
