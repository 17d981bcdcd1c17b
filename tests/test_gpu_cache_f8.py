"""GPU parity of the e4m3 cache: extend, attention of one and of many new tokens.

Extend is bit for bit: its fp32 steps are named, everything after them is a power of two
and one rounding.  Attention's tolerance, relative 2-norm against 64 bits: fp32 outputs
2e-6 (q and p of 22 bits, fp32 sums, an exponential within an ulp of an argument below
2^5: about 5 * 2^-22); bf16 and f16 outputs at most 2^-8 and 2^-11 for their own rounding
and, for many tokens, 2^-11 for the rounding of p to f16 (for one token as much again
as fp32's, which the first two hold with room)."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TOL = {"f32": 2e-6, "bf16": 2.0 ** -8 + 2.0 ** -11, "f16": 2.0 ** -10}
ONE = {"f32": 2e-6, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


@pytest.fixture(scope="module")
def ref():
    import cache_f8_reference
    return cache_f8_reference


def _case(*what):
    print("[case]", *what, file=sys.stderr, flush=True)


def _rel(x, y):
    n = np.linalg.norm(y)
    return np.linalg.norm(x - y) / (n if n else 1.0)


def _i32(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(dev)


def _first(new, start=0):
    return np.concatenate([[start], start + np.cumsum(new)]).astype(np.int32)


# ---- extend ---------------------------------------------------------------------

class Extend:
    def __init__(self, dev, ref, c, kind, heads, length, new, rot, pairs=False, pos=None, pad=0, lead=0, tail=0,
                 values=None, seed=1, in_place=False, cos=True):
        import paper_2601_07892_amd as sh
        rng = np.random.default_rng(seed)
        self.sh, self.c, self.kind, self.heads = sh, c, kind, heads
        self.length, self.first = np.asarray(length), _first(new, lead)
        self.tokens = int(self.first[-1]) + tail
        self.rot, self.pairs, self.pos, self.pad = rot, pairs, pos, pad
        t = self.tokens
        at = np.arange(c.rows)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
        self.cos, self.sin = (np.cos(at).astype(np.float32), np.sin(at).astype(np.float32)) if cos else (None, None)
        self.host, self.dev_in = {}, {}
        for name, h in (("q", heads), ("k", c.kv), ("v", c.kv)):
            x = rng.standard_normal((t, h, c.dim)).astype(np.float32) * np.exp2(rng.integers(-3, 4, (t, 1, 1)))
            if values is not None and name != "q":
                values(name, x)
            wide = torch.full((t, h * c.dim + pad), 7.0, dtype=ref.TYPES[kind])
            wide[:, :h * c.dim] = torch.from_numpy(x.astype(np.float32)).reshape(t, -1)
            self.host[name] = wide[:, :h * c.dim].float().numpy().reshape(t, h, c.dim)
            self.dev_in[name] = wide.to(dev)
        self.out = self.dev_in["q"] if in_place else torch.full_like(self.dev_in["q"], 9.0)
        self.cd = c.to(dev)
        d = self.d = sh.sherry_extend_desc()
        d.q, d.k, d.v, d.q_out = (x.data_ptr() for x in (self.dev_in["q"], self.dev_in["k"], self.dev_in["v"], self.out))
        self.df, self.dl = _i32(self.first, dev), _i32(self.length, dev)
        d.first, d.length = self.df.data_ptr(), self.dl.data_ptr()
        self.dp = None if pos is None else _i32(pos, dev)
        d.pos = ref.at(self.dp)
        if cos:
            self.dc, self.dsn = torch.from_numpy(self.cos).to(dev), torch.from_numpy(self.sin).to(dev)
            d.cos, d.sin, d.rope_rows, d.rot_dim = self.dc.data_ptr(), self.dsn.data_ptr(), c.rows, rot
        d.pairing = sh.SHERRY_ROPE_PAIRS if pairs else sh.SHERRY_ROPE_HALVES
        if pad:
            d.q_stride = d.q_out_stride = heads * c.dim + pad
            d.k_stride = d.v_stride = c.kv * c.dim + pad
        d.tokens, d.heads, d.type = t, heads, ref.CODES[kind]

    def check(self, ref, stream=None):
        from cache_reference import rotate32
        before = self.out.float().cpu().numpy()
        self.sh.sherry_cache_extend(self.cd, self.d, stream)
        torch.cuda.synchronize()
        c = self.c
        code, scale, there, where = ref.extend_plain(c, self.host, self.first, self.length, self.cos, self.sin, self.rot,
                                                     self.pairs, self.pos)
        for name in "kv":
            got, got_scale = c.read(name)
            assert np.array_equal(np.isnan(got_scale), np.isnan(scale[name]))
            assert np.array_equal(got_scale[~np.isnan(got_scale)], scale[name][~np.isnan(scale[name])])
            nan = np.isnan(ref.VALUES[code[name]])
            assert np.array_equal(np.isnan(ref.VALUES[got]), nan)
            assert np.array_equal(got[~nan], code[name][~nan])
        q = self.host["q"]
        if self.cos is not None:
            w = np.where(there, where, 0)
            q = rotate32(q, self.cos[w], self.sin[w], self.rot, self.pairs)
        q = torch.from_numpy(q).to(ref.TYPES[self.kind]).float().numpy().reshape(self.tokens, -1)
        want = before.copy()
        want[there, :q.shape[1]] = q[there]
        assert np.array_equal(self.out.float().cpu().numpy(), want)


# type, heads, kv, dim, page, rows before, new tokens
EXTENDS = [
    ("f32", 4, 2, 64, 16, [0], [1]),
    ("f32", 24, 8, 128, 16, [1, 15, 16, 17, 0, 40], [1, 1, 1, 1, 1, 1]),
    ("bf16", 8, 2, 64, 32, [0, 5, 31, 32, 33], [100, 0, 2, 64, 1]),
    ("f16", 3, 1, 256, 16, [7, 16], [9, 50]),
    ("f32", 5, 5, 80, 20, [0, 19, 21], [41, 2, 60]),
    ("bf16", 16, 2, 128, 128, [0, 100], [300, 29]),
    ("f16", 2, 2, 16, 1, [0, 3], [4, 5]),
    ("f32", 6, 3, 48, 7, [0, 6, 8], [22, 1, 13]),
    ("f32", 2, 1, 256, 200, [150, 0], [70, 130]),  # more rows than the registers keep
    ("bf16", 4, 4, 128, 64, [3] * 70, [2] * 70),    # sequences past one wave
]


@pytest.mark.parametrize("case", EXTENDS, ids=str)
@pytest.mark.parametrize("pairs", [False, True])
def test_extend(dev, ref, case, pairs):
    kind, heads, kv, dim, page, length, new = case
    _case("extend", case, pairs)
    rng = np.random.default_rng(3)
    width = max(-(-(n + m) // page) for n, m in zip(length, new)) + 1
    c = ref.Cache(rng, len(length), width, kv, page, dim, length)
    Extend(dev, ref, c, kind, heads, length, new, dim if pairs else dim // 2, pairs).check(ref)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_extend_strides_offsets_and_tokens_of_nobody(dev, ref, kind):
    rng = np.random.default_rng(4)
    c = ref.Cache(rng, 3, 6, 2, 16, 64, [5, 0, 30], extra=64)
    _case("extend strides", kind)
    # an odd padding: values one by one; tokens before first[0] and behind first[batch]
    Extend(dev, ref, c, kind, 4, [5, 0, 30], [20, 3, 9], 64, pad=3, lead=2, tail=3).check(ref)


def test_extend_in_place_without_angles_and_without_q(dev, ref):
    rng = np.random.default_rng(5)
    c = ref.Cache(rng, 2, 4, 2, 16, 64, [5, 0])
    Extend(dev, ref, c, "f32", 4, [5, 0], [20, 3], 64, in_place=True).check(ref)
    c = ref.Cache(rng, 2, 4, 2, 16, 64, [5, 0])
    Extend(dev, ref, c, "bf16", 4, [5, 0], [20, 3], 64, cos=False).check(ref)
    c = ref.Cache(rng, 2, 4, 2, 16, 64, [5, 0])
    e = Extend(dev, ref, c, "f32", 4, [5, 0], [20, 3], 64)
    e.d.q = e.d.q_out = None
    e.d.heads = 0
    e.host["q"] = e.out.cpu().numpy().reshape(e.tokens, 4, 64)
    q, e.cos_q = e.host.pop("q"), None
    before = e.out.clone()
    e.sh.sherry_cache_extend(e.cd, e.d)
    torch.cuda.synchronize()
    assert torch.equal(before, e.out)
    code, scale, _, _ = ref.extend_plain(c, e.host, e.first, e.length, e.cos, e.sin, 64, False)
    for name in "kv":
        got, got_scale = c.read(name)
        live = ~np.isnan(scale[name])
        assert np.array_equal(got_scale[live], scale[name][live])
        assert np.array_equal(got[live], code[name][live])
    del q


def test_extend_leaves_out_what_is_out_of_range(dev, ref):
    rng = np.random.default_rng(6)
    c = ref.Cache(rng, 4, 3, 2, 16, 64, [5, 40, 0, 20])
    c.table[2, 0], c.table[3, 1] = -1, c.pages  # pages that do not exist
    length, new = [5, 40, 0, 20], [4, 20, 18, 30]  # the second passes the table
    pos = np.arange(72)
    pos[[1, 45]] = [-1, c.rows]  # positions out of range
    Extend(dev, ref, c, "f32", 4, length, new, 64, pos=pos % (c.rows + 1) - (pos < 0)).check(ref)
    # lengths below 0 and past the table
    c = ref.Cache(rng, 2, 3, 2, 16, 64, [0, 48])
    Extend(dev, ref, c, "f32", 4, [-5, 1000], [4, 4], 64).check(ref)


def test_extend_values_at_the_edges(dev, ref):
    """Zeros, powers' borders (448 * 2^e and one step past it), subnormal codes, tiny and
    huge values, infinities and NaN, which do not move the power."""
    rng = np.random.default_rng(7)
    rows = [0.0, 448.0, np.nextafter(np.float32(448), np.float32(1e9)), 449.0, 1e-38, 3e38, 1e-44, 2.0 ** -9, 2.0 ** -10,
            2.0 ** -10 * 1.5, 3 * 2.0 ** -10, 17.0, 18.0, 19.0, -17.0, 464.0]

    def values(name, x):
        t = len(x)
        x[:, 0, :] = 0
        x[:, 0, :16] = np.array(rows, np.float32)[np.arange(t)[:, None] % 16]
        x[:, 1, :] = np.array(rows, np.float32)[np.arange(x.shape[2]) % 16] * (np.arange(t)[:, None] % 5 == 0)
        x[3, 1, 5], x[4, 1, 6], x[5, 1, 7] = np.inf, -np.inf, np.nan
        x[6:, 1, :] *= np.float32(2.0 ** -120)

    for page, cos in ((16, False), (1, False), (4, True)):
        _case("extend edges", page, cos)
        c = ref.Cache(rng, 1, 64 // page, 2, page, 64, [3])
        with np.errstate(all="ignore"):
            Extend(dev, ref, c, "f32", 4, [3], [40], 64, values=values, cos=cos).check(ref)


def test_extend_token_by_token_keeps_older_rows(dev, ref):
    """Rows of growing size, one call each: every row is within the steps that its
    roundings add up to of its value, and the library's codes are the plain ones'."""
    rng = np.random.default_rng(8)
    c = ref.Cache(rng, 1, 2, 1, 16, 64, [0])
    first = {n: [] for n in "kv"}
    for i in range(20):
        e = Extend(dev, ref, c, "f32", 2, [i], [1], 64, cos=False, seed=20 + i,
                   values=lambda name, x, i=i: np.multiply(x, np.float32(2.0 ** (i % 7)), out=x))
        e.check(ref)
        for name in "kv":
            first[name].append(e.host[name][0, 0].astype(np.float64))
            c.code[name], c.scale[name] = c.read(name)
    for name in "kv":
        got, _ = c.rows64(name, 0, 0, 20)
        power = np.repeat(c.power(name)[c.table[0], 0], 16)[:20, None]
        x = np.array(first[name])
        # a rounding is off by 2^-4 of a normal value, half a step of 2^-9 of a subnormal one;
        # the steps double with the power, and so add up to less than twice the last
        assert np.all(np.abs(got - x) <= 2 * (2.0 ** -4 * np.abs(x) + 2.0 ** -10 * power))


@pytest.mark.parametrize("kind,heads,dim", [("bf16", 20, 64), ("f32", 40, 128)])
def test_extend_of_so_many_tokens_that_workgroups_turn_several(dev, ref, kind, heads, dim):
    """q of tokens that a workgroup takes one after the other: sequences that end among them,
    that have none, and tokens that belong to nobody or lie past the table."""
    _case("extend many", kind, heads, dim)
    length, new = [3, 0, 16, 700, 5, 9, 40, 990], [700, 0, 1, 300, 3, 2, 1100, 60]
    c = ref.Cache(np.random.default_rng(19), 8, 64, 1, 16, dim, length)
    Extend(dev, ref, c, kind, heads, length, new, dim, lead=5, tail=9).check(ref)


# ---- attention ------------------------------------------------------------------

class Attend:
    def __init__(self, dev, ref, c, kind, heads, length, new, window=0, mask=None, scale=None, pad=0, lead=0, tail=0, q=None):
        import paper_2601_07892_amd as sh
        rng = np.random.default_rng(11)
        self.sh, self.c, self.kind, self.heads, self.window, self.mask = sh, c, kind, heads, window, mask
        self.length, self.first = np.asarray(length), _first(new, lead)
        self.tokens = int(self.first[-1]) + tail
        self.scale = float(np.float32(c.dim ** -0.5 if scale is None else scale))
        row = heads * c.dim
        q = rng.standard_normal((self.tokens, heads, c.dim)) * 2 if q is None else q
        wide = torch.zeros((self.tokens, row + pad), dtype=ref.TYPES[kind])
        wide[:, :row] = torch.from_numpy(q.astype(np.float32)).reshape(self.tokens, -1)
        self.q = wide[:, :row].float().numpy().reshape(q.shape)
        self.qd = wide.to(dev)
        self.out = torch.full((self.tokens, row + pad), 9.0, dtype=ref.TYPES[kind], device=dev)
        self.cd = c.to(dev)
        d = self.d = sh.sherry_attend_tokens_desc()
        self.df, self.dl = _i32(self.first, dev), _i32(self.length, dev)
        self.dm = None if mask is None else torch.from_numpy(np.ascontiguousarray(mask, np.uint8)).to(dev)
        d.q, d.out, d.first, d.length = (x.data_ptr() for x in (self.qd, self.out, self.df, self.dl))
        d.mask, d.mask_stride = ref.at(self.dm), mask.shape[1] if mask is not None else 0
        d.q_stride = d.out_stride = row + pad
        d.tokens, d.heads, d.type, d.window, d.scale = self.tokens, heads, ref.CODES[kind], window, self.scale
        n = sh.sherry_cache_attend_tokens_workspace(self.cd, d)
        assert n > 0
        self.ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=dev)
        d.workspace, d.workspace_bytes = self.ws.data_ptr(), n

    def run(self, stream=None):
        self.sh.sherry_cache_attend_tokens(self.cd, self.d, stream)
        torch.cuda.synchronize()
        assert bool((self.ws[-64:] == 0xFF).all())
        row = self.heads * self.c.dim
        assert bool((self.out[:, row:] == 9.0).all())
        return self.out[:, :row].double().cpu().numpy().reshape(self.tokens, self.heads, self.c.dim)

    def check(self, ref, stream=None):
        got = self.run(stream)
        want = ref.attend64(self.c, self.q, self.first, self.length, self.scale, self.window, self.mask)
        nobody = np.ones(self.tokens, bool)
        for b in range(self.c.batch):
            s = slice(self.first[b], self.first[b + 1])
            nobody[s] = False
            if self.first[b] == self.first[b + 1]:
                continue
            assert np.all(np.isfinite(got[s])), b
            assert _rel(got[s], want[s]) <= TOL[self.kind], (b, _rel(got[s], want[s]))
            for t in range(self.first[b], self.first[b + 1]):  # no token's error hides behind the others'
                assert _rel(got[t], want[t]) <= 4 * TOL[self.kind], (b, t)
        assert np.all(got[nobody] == 9.0)
        empty = ~nobody & np.all(want == 0, axis=(1, 2))
        assert np.all(got[empty] == 0)
        return got


# type, heads, kv, dim, page, rows before, new tokens
TOKENS = [
    ("f32", 4, 1, 64, 16, [0], [1]),
    ("f32", 8, 2, 64, 16, [0, 63, 64, 65], [3, 1, 2, 1]),
    ("bf16", 8, 2, 128, 32, [0, 100], [70, 33]),
    ("f16", 6, 2, 64, 16, [0, 0, 500], [1, 130, 40]),
    ("f32", 6, 2, 128, 64, [10, 0, 7], [65, 0, 128]),
    ("bf16", 3, 3, 256, 16, [0, 31], [66, 5]),
    ("f32", 2, 1, 256, 32, [200], [40]),
    ("f16", 5, 1, 80, 20, [0, 19, 300], [50, 2, 21]),
    ("bf16", 40, 2, 64, 128, [300, 0], [7, 20]),
    ("f32", 3, 1, 48, 7, [100, 3], [9, 30]),
    ("bf16", 200, 1, 64, 16, [40], [3]),           # more heads than a tile has rows
    ("bf16", 256, 2, 16, 1, [5, 70], [2, 1]),
    ("f16", 64, 1, 128, 16, [0] * 70, [2] * 70),    # sequences past one wave
]


@pytest.mark.parametrize("case", TOKENS, ids=str)
def test_tokens(dev, ref, case):
    kind, heads, kv, dim, page, length, new = case
    _case("tokens", case)
    full = [n + m for n, m in zip(length, new)]
    c = ref.Cache(np.random.default_rng(9), len(length), max(-(-n // page) for n in full) + 1, kv, page, dim, full)
    Attend(dev, ref, c, kind, heads, length, new).check(ref)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 20), (256, 64)])
@pytest.mark.parametrize("window", [0, 1, 37, 64, 1000])
def test_tokens_windows_masks_and_absent_pages(dev, ref, kind, dim, page, window):
    _case("tokens masks", kind, dim, page, window)
    rng = np.random.default_rng(10)
    length, new = [150, 0, 3, 64], [40, 70, 1, 64]
    full = [n + m for n, m in zip(length, new)]
    width = -(-max(full) // page) + 1
    c = ref.Cache(rng, 4, width, 2, page, dim, full)
    mask = (rng.random((4, width * page + 3)) < 0.8).astype(np.uint8)
    mask[1, :30] = 0       # the first tokens of a prompt: nothing
    mask[2] = 0            # a sequence: nothing
    c.table[0, 1], c.table[3, 0], c.table[3, 2] = -1, c.pages, -7
    # rows that are left out hold NaN
    for b in range(4):
        for r in range(min(full[b], c.rows)):
            p = c.table[b, r // page]
            if not mask[b, r] and 0 <= p < c.pages:
                c.code["k"][p, :, r % page] = 0x7F
                c.code["v"][p, :, r % page] = 0xFF
    Attend(dev, ref, c, kind, 6, length, new, window=window, mask=mask, pad=8, lead=1, tail=2).check(ref)


def test_tokens_nan_reaches_only_the_tokens_that_attend_to_it(dev, ref):
    for kind in ("f32", "bf16"):
        for name, window in (("v", 0), ("k", 0), ("v", 20), ("k", 20)):
            _case("tokens nan", kind, name, window)
            c = ref.Cache(np.random.default_rng(12), 1, 9, 1, 16, 64, [140])
            row = 100
            c.code[name][c.table[0, row // 16], 0, row % 16, 5] = 0x7F
            a = Attend(dev, ref, c, kind, 4, [60], [80], window=window)
            got = a.run()
            tokens = np.arange(60, 140)
            hit = (tokens >= row) & ((tokens < row + window) if window else True)
            bad = np.isnan(got)
            if name == "k":
                assert np.array_equal(bad.any((1, 2)), hit) and bad[hit].all()
            else:
                assert bad[hit][..., 5].all() and bad.sum() == hit.sum() * 4
            with np.errstate(invalid="ignore"):
                want = ref.attend64(c, a.q, a.first, a.length, a.scale, window)
            assert _rel(got[~bad], want[~bad]) <= TOL[kind]


def test_tokens_long_rows_are_split_and_joined(dev, ref):
    """Few tokens over many rows: their tiles are cut over workgroups."""
    rng = np.random.default_rng(13)
    for kind, heads, kv, dim, length, new in (("f32", 4, 1, 64, [9000], [1]), ("bf16", 8, 2, 128, [5000, 1], [3, 2]),
                                              ("f16", 4, 4, 256, [3000, 0, 2000], [2, 5, 1])):
        _case("tokens split", kind, dim, length)
        full = [n + m for n, m in zip(length, new)]
        c = ref.Cache(rng, len(length), -(-max(full) // 32), kv, 32, dim, full)
        Attend(dev, ref, c, kind, heads, length, new).check(ref)
        # with nothing to attend to but in the middle
        mask = np.zeros((len(length), c.rows), np.uint8)
        mask[0, 1500:1503] = 1
        Attend(dev, ref, c, kind, heads, length, new, mask=mask).check(ref)


@pytest.mark.parametrize("kind,dim,page", [("f32", 64, 16), ("bf16", 64, 48), ("bf16", 128, 10), ("f16", 256, 32)])
@pytest.mark.parametrize("window", [0, 130])
def test_tokens_over_every_number_of_blocks(dev, ref, kind, dim, page, window):
    """Tiles over 1 to 11 blocks of rows, ending at, before and behind a block's end, with rows
    left out that hold NaN."""
    _case("tokens blocks", kind, dim, page, window)
    rng = np.random.default_rng(20)
    length = [max(0, 64 * i + j) for i in range(1, 12) for j in (-2, -1, 0)]
    new = [1 + i % 3 for i in range(len(length))]
    full = [n + m for n, m in zip(length, new)]
    c = ref.Cache(rng, len(length), -(-max(full) // page), 1, page, dim, full)
    mask = (rng.random((len(length), c.rows)) < 0.95).astype(np.uint8)
    mask[::2] = 1
    for b in range(len(length)):
        for r in np.flatnonzero(mask[b, :full[b]] == 0):
            c.code["k"][c.table[b, r // page], :, r % page] = 0x7F
            c.code["v"][c.table[b, r // page], :, r % page] = 0xFF
    Attend(dev, ref, c, kind, 3, length, new, window=window, mask=mask).check(ref)


@pytest.mark.parametrize("kind,heads,kv,dim,window", [("bf16", 4, 1, 128, 0), ("f32", 4, 2, 64, 0), ("f16", 2, 1, 256, 0),
                                                      ("bf16", 6, 2, 64, 777)])
def test_tokens_whose_tiles_many_workgroups_share(dev, ref, kind, heads, kv, dim, window):
    """Runs that end inside tiles, near their begin and near their end, several a tile."""
    _case("tokens shared tiles", kind, heads, kv, dim, window)
    length, new = [3000, 0, 1500], [200, 333, 70]
    full = [n + m for n, m in zip(length, new)]
    c = ref.Cache(np.random.default_rng(21), 3, -(-max(full) // 16), kv, 16, dim, full, spread=6)
    Attend(dev, ref, c, kind, heads, length, new, window=window).check(ref)


@pytest.mark.parametrize("kind,every", [("f32", 1), ("bf16", 3), ("f32", 130)])
def test_tokens_of_many_sequences_most_of_them_without(dev, ref, kind, every):
    """Workgroups that go on from sequence to sequence, over those without tokens."""
    _case("tokens many sequences", kind, every)
    rng = np.random.default_rng(22)
    length = [int(n) for n in rng.integers(0, 150, 300)]
    new = [1 + i % 4 if i % every == every // 2 else 0 for i in range(300)]
    full = [n + m for n, m in zip(length, new)]
    c = ref.Cache(rng, 300, -(-max(full) // 16), 1, 16, 64, full)
    Attend(dev, ref, c, kind, 2, length, new, lead=1, tail=2).check(ref)


@pytest.mark.parametrize("scale", [0.0, -0.2, 30.0, 1e-30])
def test_tokens_scales_of_scores(dev, ref, scale):
    """No, negative, one-hot and vanishing scores; powers of pages far apart."""
    c = ref.Cache(np.random.default_rng(14), 2, 8, 2, 16, 64, [128, 60], spread=12)
    a = Attend(dev, ref, c, "f32", 4, [90, 0], [38, 60], scale=scale)
    got = a.run()
    want = ref.attend64(c, a.q, a.first, a.length, a.scale)
    # (scores to 2^10 times an error of 2^-22 of the largest terms: exponents off by 2^-12 at most)
    assert _rel(got, want) <= (2.0 ** -11 if scale == 30.0 else TOL["f32"])


def test_tokens_scores_rise_and_fall(dev, ref):
    """A maximum that rises from block to block, and one that is met at once: sums are
    rescaled, or never again."""
    for up in (True, False):
        c = ref.Cache(np.random.default_rng(15), 1, 20, 1, 16, 64, [320])
        for r in range(320):
            j = r if up else 319 - r
            c.scale["k"][c.table[0, r // 16], 0] = 2.0 ** (j // 16 // 4 - 6)
            c.scale["v"][c.table[0, r // 16], 0] = 2.0 ** (j // 16 // 2 - 9)
        Attend(dev, ref, c, "f32", 4, [300], [20]).check(ref)


def test_tokens_past_the_table(dev, ref):
    """Tokens whose row lies past the table attend to all of it."""
    c = ref.Cache(np.random.default_rng(16), 2, 3, 1, 16, 64, [48, 48])
    Attend(dev, ref, c, "f32", 2, [40, 1000], [20, 5]).check(ref)
    Attend(dev, ref, c, "f32", 2, [40, 1000], [20, 5], window=30).check(ref)


# ---- one token: the e4m3 form of the attention that other caches have ------------

@pytest.mark.parametrize("kind,heads,kv,dim,page,lens", [
    ("f32", 8, 2, 64, 16, [1]), ("f32", 8, 8, 128, 16, [31, 32, 33, 0, 1]), ("bf16", 12, 4, 128, 64, [130, 15, 700]),
    ("f16", 6, 2, 64, 48, [100, 49, 1]), ("f32", 4, 1, 256, 16, [65, 1000]), ("f16", 9, 3, 80, 20, [95, 96, 97]),
    ("bf16", 40, 2, 256, 16, [77, 160]), ("f32", 5, 5, 48, 7, [50, 3]), ("bf16", 16, 1, 16, 1, [5, 2000])])
@pytest.mark.parametrize("window,masked", [(0, False), (40, True)])
def test_one_token(dev, ref, kind, heads, kv, dim, page, lens, window, masked):
    import paper_2601_07892_amd as sh
    _case("one token", kind, heads, kv, dim, page, lens, window, masked)
    rng = np.random.default_rng(17)
    batch, width = len(lens), -(-max(lens) // page) + 1
    c = ref.Cache(rng, batch, width, kv, page, dim, lens, spread=8)
    cd = c.to(dev)
    q = torch.from_numpy(rng.standard_normal((batch, heads, dim)) * 2).to(ref.TYPES[kind])
    mask = (rng.random((batch, c.rows)) < 0.7).astype(np.uint8) if masked else None
    qd, out, dl = q.to(dev), torch.empty_like(q, device=dev), _i32(lens, dev)
    dm = None if mask is None else torch.from_numpy(mask).to(dev)
    weight = torch.zeros((batch, kv, c.rows), device=dev) if masked else None
    d = sh.sherry_attend_desc()
    d.q, d.out, d.length, d.mask, d.mask_stride = qd.data_ptr(), out.data_ptr(), dl.data_ptr(), ref.at(dm), c.rows
    d.heads, d.type, d.window, d.scale = heads, ref.CODES[kind], window, dim ** -0.5
    d.weight, d.row_stride = ref.at(weight), c.rows
    n = sh.sherry_cache_attend_workspace(cd, d)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=dev)
    d.workspace, d.workspace_bytes = ws.data_ptr(), n
    sh.sherry_cache_attend(cd, d)
    torch.cuda.synchronize()
    got = out.double().cpu().numpy()
    some = np.array(lens) > 0
    first = _first(some.astype(int))
    want = np.zeros(got.shape)
    want[some] = ref.attend64(c, q.float().numpy()[some], first, np.array(lens) - 1, float(np.float32(dim ** -0.5)), window, mask)
    assert np.all(np.isfinite(got)) and _rel(got, want) <= ONE[kind]
    for b in range(batch):
        assert _rel(got[b], want[b]) <= 4 * ONE[kind], b
    if weight is not None:  # probabilities of a token add up to one per query head
        total = weight.double().sum(-1).cpu().numpy()
        some = np.array([[mask[b, max(0, lens[b] - window):lens[b]].any()] * kv for b in range(batch)])
        assert np.allclose(total, some * (heads // kv), rtol=1e-5, atol=0)


# ---- together ---------------------------------------------------------------------

def test_prompt_in_chunks_then_tokens(dev, ref):
    """A prompt in two chunks and tokens one by one: every step's attention over what
    extend has stored, and the one-token form against the same."""
    import paper_2601_07892_amd as sh
    rng = np.random.default_rng(18)
    c = ref.Cache(rng, 2, 6, 2, 16, 64, [0, 0])
    length = np.zeros(2, int)
    for new in ([30, 17], [20, 33], [1, 1], [1, 1]):
        _case("chunks", list(length), new)
        e = Extend(dev, ref, c, "bf16", 4, length, new, 64, seed=int(length.sum()))
        e.check(ref)
        for name in "kv":
            c.code[name], c.scale[name] = c.read(name)
        q = e.out.float().cpu().numpy().reshape(e.tokens, 4, 64)
        a = Attend(dev, ref, c, "bf16", 4, length, new, q=q)
        got = a.check(ref)
        length = length + new
        if new == [1, 1]:
            d, dl = sh.sherry_attend_desc(), _i32(length, dev)
            out = torch.empty((2, 256), dtype=torch.bfloat16, device=dev)
            d.q, d.out, d.length = a.qd.data_ptr(), out.data_ptr(), dl.data_ptr()
            d.heads, d.type, d.scale = 4, sh.SHERRY_BF16, a.scale
            n = sh.sherry_cache_attend_workspace(a.cd, d)
            ws = torch.empty(n, dtype=torch.uint8, device=dev)
            d.workspace, d.workspace_bytes = ws.data_ptr(), n
            sh.sherry_cache_attend(a.cd, d)
            torch.cuda.synchronize()
            assert _rel(out.double().cpu().numpy().reshape(got.shape), got) <= 2 * TOL["bf16"]


def test_captured_and_on_another_stream(dev, ref):
    """extend and attention of its tokens in a graph, replayed with new lengths and
    inputs and eager work between; and on a stream of their own."""
    rng = np.random.default_rng(19)
    c = ref.Cache(rng, 2, 6, 2, 16, 64, [0, 0])
    e = Extend(dev, ref, c, "f32", 4, [0, 0], [9, 9], 64)
    code, scale = {n: e.c.d[n].clone() for n in "kv"}, {n: e.c.ds[n].clone() for n in "kv"}
    # (the cache's buffers are now those that the attention's harness has made)
    a = Attend(dev, ref, c, "f32", 4, [0, 0], [9, 9])
    e.cd, a.d.length, a.d.first, a.d.q = a.cd, e.d.length, e.d.first, e.d.q_out
    a.d.q_stride = a.d.out_stride = 0
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        e.sh.sherry_cache_extend(e.cd, e.d)
        a.sh.sherry_cache_attend_tokens(a.cd, a.d)

    def restart():
        for n in "kv":
            c.d[n].copy_(code[n])
            c.ds[n].copy_(scale[n])

    results = {}
    for how in ("graph", "eager", "stream"):
        for length in ([0, 0], [20, 3], [60, 87]):
            restart()
            e.dl.copy_(_i32(length, dev))
            a.out.zero_()
            torch.cuda.synchronize()
            if how == "graph":
                graph.replay()
            elif how == "eager":
                e.sh.sherry_cache_extend(e.cd, e.d)
                a.sh.sherry_cache_attend_tokens(a.cd, a.d)
            else:
                e.sh.sherry_cache_extend(e.cd, e.d, side)
                a.sh.sherry_cache_attend_tokens(a.cd, a.d, side)
            torch.cuda.synchronize()
            got = [a.out.clone()] + [c.d[n].clone() for n in "kv"] + [c.ds[n].clone() for n in "kv"]
            key = tuple(length)
            if key in results:
                for x, y in zip(got, results[key]):
                    assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float())), (how, length)
            else:
                results[key] = got
