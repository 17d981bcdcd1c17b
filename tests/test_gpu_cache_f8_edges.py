"""GPU tests of the e4m3 cache where its calls are easily wrong."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_cache_f8 import TOL, Attend, Extend, _case, _i32, _rel, dev, ref  # noqa: E402, F401


def _check_each(a, got, want, tokens, tol):
    for t in tokens:
        assert np.all(np.isfinite(got[t])), t
        assert _rel(got[t], want[t]) <= tol, (t, _rel(got[t], want[t]))


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


# ---- powers far apart --------------------------------------------------------------

def _powers(c, b, name, exponent):
    """Sets the exponents of sequence b's pages, one a page of its table."""
    for j, e in enumerate(exponent):
        c.scale[name][c.table[b, j]] = np.float32(2.0 ** int(e))


@pytest.mark.parametrize("kind,base,up", [("f32", -14, 20), ("bf16", -14, 20), ("f16", -14, 20), ("f32", -30, 45), ("bf16", -90, 150)])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 7), (256, 32)])
@pytest.mark.parametrize("window", [0, 40])
def test_tokens_v_of_rows_that_a_token_leaves_out(dev, ref, kind, base, up, dim, page, window):
    """V far larger in rows behind a token, or before its window, than in the rows that it attends to."""
    _case("tokens v powers", kind, base, up, dim, page, window)
    n, new = 230, 170
    c = ref.Cache(np.random.default_rng(31), 1, -(-n // page), 2, page, dim, [n])
    at = np.arange(c.width) * page
    _powers(c, 0, "v", base + up * ((at < 100) if window else (at >= 130)))
    a = Attend(dev, ref, c, kind, 6, [n - new], [new], window=window)
    got, want = a.run(), ref.attend64(c, a.q, a.first, a.length, a.scale, window)
    _check_each(a, got, want, range(new), 4 * TOL[kind])


@pytest.mark.parametrize("kind,up", [("f32", 18), ("bf16", 30), ("f32", 120), ("f16", 50)])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 10), (256, 32)])
@pytest.mark.parametrize("window", [0, 40])
def test_tokens_k_of_rows_that_a_token_leaves_out(dev, ref, kind, up, dim, page, window):
    """K far larger in rows that some tokens leave out: what these get (the others' scores pass what
    fp32 tells apart)."""
    _case("tokens k powers", kind, up, dim, page, window)
    n, new = 230, 170
    c = ref.Cache(np.random.default_rng(32), 1, -(-n // page), 2, page, dim, [n])
    at = np.arange(c.width) * page
    big = (at < 100) if window else (at >= 130)
    _powers(c, 0, "k", -6 + up * big)
    a = Attend(dev, ref, c, kind, 6, [n - new], [new], window=window)
    got = a.run()
    with np.errstate(over="ignore", invalid="ignore"):
        want = ref.attend64(c, a.q, a.first, a.length, a.scale, window)
    rows = np.flatnonzero(np.repeat(big, page)[:n])
    own = n - new + np.arange(new)
    free = [t for t in range(new) if not np.any((rows <= own[t]) & ((rows > own[t] - window) | (window == 0)))]
    assert len(free) > 20
    _check_each(a, got, want, free, 4 * TOL[kind])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page,window", [(64, 16, 0), (64, 5, 90), (128, 20, 0), (128, 64, 300), (256, 16, 70)])
def test_tokens_over_pages_of_any_powers(dev, ref, kind, dim, page, window):
    """Powers from page to page anywhere, masks, absent pages, NaN in rows that are left out, pages
    of zeros (whose power is the smallest that extend gives), runs that end inside tiles."""
    _case("tokens any powers", kind, dim, page, window)
    rng = np.random.default_rng(33)
    length, new = [0, 500, 3, 1100], [150, 40, 1, 5]
    full = [n + m for n, m in zip(length, new)]
    c = ref.Cache(rng, 4, -(-max(full) // page), 2, page, dim, full)
    for b in range(4):
        _powers(c, b, "v", rng.integers(-60, 20, c.width))
        _powers(c, b, "k", rng.integers(-45, -5, c.width))
    for b, j in ((0, 2), (1, 0), (3, 7)):
        for name in "kv":
            c.code[name][c.table[b, j]] &= 0x80
            c.scale[name][c.table[b, j]] = 2.0 ** -100
    mask = (rng.random((4, c.rows)) < 0.9).astype(np.uint8)
    for b in range(4):
        for r in np.flatnonzero(mask[b, :full[b]] == 0):
            c.code["k"][c.table[b, r // page], :, r % page] = 0x7F
            c.code["v"][c.table[b, r // page], :, r % page] = 0xFF
    c.table[1, 3] = -1
    Attend(dev, ref, c, kind, 6, length, new, window=window, mask=mask).check(ref)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_tokens_nan_on_pages_of_powers_far_apart(dev, ref, kind):
    """As where the powers are near: NaN in V reaches its value of the tokens that attend to the row,
    and no others."""
    for window in (0, 20):
        _case("tokens nan, powers", kind, window)
        c = ref.Cache(np.random.default_rng(34), 1, 9, 1, 16, 64, [140])
        _powers(c, 0, "v", [-5, 30, -40, 7, -5, -6, 20, 0, 1])
        row = 100
        c.code["v"][c.table[0, row // 16], 0, row % 16, 5] = 0x7F
        a = Attend(dev, ref, c, kind, 4, [60], [80], window=window)
        got = a.run()
        tokens = np.arange(60, 140)
        hit = (tokens >= row) & ((tokens < row + window) if window else True)
        bad = np.isnan(got)
        assert bad[hit][..., 5].all() and bad.sum() == hit.sum() * 4
        with np.errstate(invalid="ignore"):
            want = ref.attend64(c, a.q, a.first, a.length, a.scale, window)
        _check_each(a, got, want, np.flatnonzero(~hit), 4 * TOL[kind])


# ---- f16 outputs -------------------------------------------------------------------

@pytest.mark.parametrize("heads,kv,dim,length,new,window", [
    (4, 1, 64, [0], [200], 0), (6, 2, 128, [30, 700], [130, 40], 0), (2, 1, 256, [300], [60], 0), (4, 2, 64, [2500, 40], [5, 90], 64)], ids=str)
def test_tokens_f16_outputs_are_rounded_once(dev, ref, heads, kv, dim, length, new, window):
    """The output's own rounding is all that an f16 output loses beside what an fp32 output does.
    With y the unrounded output, |y - want| <= 2e-6 |want| (as fp32 outputs are held to), and the distance
    to the nearest f16 value changes by no more than its argument:
    |f16(y) - want| <= |f16(y) - y| + |y - want| <= |f16(want) - want| + 2 |y - want|."""
    _case("tokens f16", heads, kv, dim, length, new, window)
    full = [n + m for n, m in zip(length, new)]
    c = ref.Cache(np.random.default_rng(35), len(full), -(-max(full) // 16), kv, 16, dim, full)
    a = Attend(dev, ref, c, "f16", heads, length, new, window=window)
    got, want = a.run(), ref.attend64(c, a.q, a.first, a.length, a.scale, window)
    least = np.linalg.norm(want.astype(np.float16).astype(np.float64) - want)
    assert np.linalg.norm(got - want) <= least + 4e-6 * np.linalg.norm(want)


# ---- extend: tokens left out, the largest power ---------------------------------------

def _bytes(c):
    return {n: (c.d[n].cpu().numpy().copy(), c.ds[n].cpu().numpy().view(np.uint32).copy()) for n in "kv"}


@pytest.mark.parametrize("page,new,kv", [(16, 3, 2), (16, 40, 5), (128, 200, 1)])
def test_extend_leaves_pages_alone_that_get_no_rows(dev, ref, page, new, kv):
    """Every token's position is out of range: no code and no power changes, of a page that holds
    rows (with a power below the least that extend gives) and of one that holds none."""
    for n in (5, 0):
        _case("extend nothing stored", page, new, kv, n)
        c = ref.Cache(np.random.default_rng(36), 1, 4, kv, page, 64, [n])
        for name in "kv":
            if n:
                c.scale[name][c.table[0, 0]] = 2.0 ** -110
            c.scale[name][c.table[0, 1:]] = 0.375
        e = Extend(dev, ref, c, "f32", 4, [n], [new], 64, pos=[-1 - i for i in range(new)])
        before, q = _bytes(c), e.out.clone()
        e.sh.sherry_cache_extend(e.cd, e.d)
        torch.cuda.synchronize()
        after = _bytes(c)
        for name in "kv":
            assert np.array_equal(before[name][0], after[name][0]) and np.array_equal(before[name][1], after[name][1])
        assert torch.equal(q, e.out)


@pytest.mark.parametrize("page,new", [(16, 6), (64, 50), (128, 100)])
def test_extend_rounds_rows_of_tokens_left_out_as_the_page_s_others(dev, ref, page, new):
    """The power of a page that holds rows rises: every row that gets no new codes follows it, the
    rows of tokens that are left out too."""
    _case("extend left out", page, new)
    rng = np.random.default_rng(37)
    c = ref.Cache(rng, 1, 2, 2, page, 64, [page])
    for name in "kv":
        c.scale[name][c.table[0, 0]] = 2.0 ** -6
    n = 7
    pos = np.arange(n, n + new)
    out = np.arange(new) % 3 == 1
    pos[out] = -1
    e = Extend(dev, ref, c, "f32", 2, [n], [new], 64, pos=pos, cos=True,
               values=lambda name, x: np.multiply(x, np.float32(64), out=x))
    e.sh.sherry_cache_extend(e.cd, e.d)
    torch.cuda.synchronize()
    stored = np.zeros(page, bool)
    stored[[n + i for i in range(new) if not out[i] and n + i < page]] = True
    p = c.table[0, 0]
    for name in "kv":
        code, scale = c.read(name)
        for h in range(2):
            ratio = 2.0 ** -6 / float(scale[p, h])
            assert ratio < 1
            want = ref.encode(ref.VALUES[c.code[name][p, h]] * ratio)
            assert np.array_equal(code[p, h][~stored], want[~stored])


@pytest.mark.parametrize("old", [2.0 ** 127, 2.0 ** 126, float("inf")])
@pytest.mark.parametrize("page", [16, 128])
def test_extend_into_pages_of_the_largest_power(dev, ref, old, page):
    """A page's power of 2^127 (an infinity counts as that) stays, and values near fp32's largest are
    codes about 1 of it."""
    _case("extend largest power", old, page)

    def values(name, x):
        x[:] = np.float32(3e38) * np.random.default_rng(38).uniform(-1, 1, x.shape).astype(np.float32)

    c = ref.Cache(np.random.default_rng(39), 1, 1, 2, page, 64, [3])
    for name in "kv":
        c.scale[name][c.table[0, 0]] = old
    with np.errstate(all="ignore"):
        Extend(dev, ref, c, "f32", 2, [3], [9], 64, values=values, cos=False).check(ref)
    code, scale = c.read("v")
    assert np.all(scale[c.table[0, 0]] == min(old, 2.0 ** 127)) and np.any(ref.VALUES[code[c.table[0, 0], :, 3:12]] != 0)


# ---- replays with new lengths, against the plain references -----------------------------

def test_replays_with_new_lengths_give_what_the_references_do(dev, ref):
    """extend and attention of its tokens in one graph, under fixed descriptors and workspace:
    every replay's codes, powers and outputs against the references, with eager work between."""
    rng = np.random.default_rng(40)
    c = ref.Cache(rng, 2, 40, 2, 16, 64, [640, 640])
    e = Extend(dev, ref, c, "f32", 4, [0, 0], [9, 9], 64)
    a = Attend(dev, ref, c, "f32", 4, [0, 0], [9, 9])
    e.cd, a.d.length, a.d.first, a.d.q = a.cd, e.d.length, e.d.first, e.d.q_out
    a.d.q_stride = a.d.out_stride = 0
    code, scale = {n: c.d[n].clone() for n in "kv"}, {n: c.ds[n].clone() for n in "kv"}
    start = {n: (c.code[n].copy(), c.scale[n].copy()) for n in "kv"}
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        e.sh.sherry_cache_extend(e.cd, e.d)
        a.sh.sherry_cache_attend_tokens(a.cd, a.d)
    for length in ([0, 0], [600, 3], [20, 631], [1, 0], [600, 3]):
        _case("replay", length)
        for n in "kv":
            c.code[n], c.scale[n] = start[n][0].copy(), start[n][1].copy()
            c.d[n].copy_(code[n])
            c.ds[n].copy_(scale[n])
        e.length = np.array(length)
        e.dl.copy_(_i32(length, dev))
        e.out.fill_(9.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, powers, there, _ = ref.extend_plain(c, e.host, e.first, e.length, e.cos, e.sin, 64, False)
        assert there.all()
        for n in "kv":
            got, got_scale = c.read(n)
            assert np.array_equal(got, want[n]) and np.array_equal(got_scale, powers[n], equal_nan=True)
            c.code[n], c.scale[n] = got, got_scale
        q = e.out.float().cpu().numpy().reshape(18, 4, 64)
        out = a.out.double().cpu().numpy().reshape(18, 4, 64)
        _check_each(a, out, ref.attend64(c, q, e.first, e.length, a.scale), range(18), 4 * TOL["f32"])


# ---- strides and pools beyond 2^31 bytes ------------------------------------------------

def _far_apart(c, dev):
    """c.to(dev) with its pages so far from each other that the pools pass 2^31 bytes."""
    import paper_2601_07892_amd as sh
    whole = c.kv * c.page * c.dim
    small = c.stride
    c.stride = whole
    cd = c.to(dev)
    c.stride = ((2 ** 31 // (c.pages - 1)) // 16 + 1) * 16
    for n in "kv":
        far = torch.zeros(c.pages * c.stride, dtype=torch.uint8, device=dev)
        far.view(c.pages, c.stride)[:, :whole] = c.d[n]
        c.d[n] = far
    cd.k, cd.v, cd.page_stride = c.d["k"].data_ptr(), c.d["v"].data_ptr(), c.stride
    assert cd.type == sh.SHERRY_F8 and (c.pages - 1) * c.stride >= 2 ** 31 and small == whole
    return cd


def test_pools_beyond_31_bits(dev, ref):
    """extend, attention of many tokens and of one, over pages up to 2^31 bytes and more from the pool's start."""
    import paper_2601_07892_amd as sh
    _case("far pages")
    c = ref.Cache(np.random.default_rng(41), 2, 4, 2, 16, 64, [30, 9])
    c.table[0, 0], c.table[1, 0] = c.pages - 1, c.pages - 2  # (taken from no other place)
    spare = [p for p in range(c.pages - 2) if p not in set(c.table.ravel())]
    seen = set()
    for i in np.ndindex(*c.table.shape):  # every page once
        if int(c.table[i]) in seen:
            c.table[i] = spare.pop()
        seen.add(int(c.table[i]))
    for name in "kv":
        c.code[name] = ref.encode(np.random.default_rng(42).standard_normal(c.code[name].shape) * 40)
        c.scale[name][:] = 2.0 ** -6
    e = Extend(dev, ref, c, "f32", 4, [30, 9], [20, 12], 64)
    e.cd = _far_apart(c, dev)
    want, powers, _, _ = ref.extend_plain(c, e.host, e.first, e.length, e.cos, e.sin, 64, False)
    sh.sherry_cache_extend(e.cd, e.d)
    torch.cuda.synchronize()
    whole = c.kv * c.page * c.dim
    for n in "kv":
        got = c.d[n].view(c.pages, c.stride)[:, :whole].cpu().numpy().reshape(c.code[n].shape)
        assert np.array_equal(got, want[n]) and np.array_equal(c.ds[n].cpu().numpy(), powers[n])
        c.code[n], c.scale[n] = got, powers[n]
    pools, scales, table = dict(c.d), dict(c.ds), c.dt  # (the harness below makes others)
    c.stride = whole
    a = Attend(dev, ref, c, "f32", 4, [30, 9], [20, 12])
    a.cd = e.cd
    c.d, c.ds = pools, scales
    a.check(ref)
    assert table.data_ptr() == e.cd.table
    d, out = sh.sherry_attend_desc(), torch.empty((2, 256), device=dev)
    q = torch.from_numpy(np.random.default_rng(43).standard_normal((2, 4, 64)).astype(np.float32))
    qd, dl = q.to(dev), _i32([50, 21], dev)
    d.q, d.out, d.length, d.heads, d.type, d.scale = qd.data_ptr(), out.data_ptr(), dl.data_ptr(), 4, sh.SHERRY_F32, 0.125
    n = sh.sherry_cache_attend_workspace(e.cd, d)
    ws = torch.empty(n, dtype=torch.uint8, device=dev)
    d.workspace, d.workspace_bytes = ws.data_ptr(), n
    sh.sherry_cache_attend(e.cd, d)
    torch.cuda.synchronize()
    first = np.array([0, 1, 2])
    want = ref.attend64(c, q.numpy(), first, np.array([49, 20]), 0.125)
    _check_each(a, out.double().cpu().numpy().reshape(2, 4, 64), want, range(2), 4 * TOL["f32"])


@pytest.mark.parametrize("kind,dim,page,extra", [("f32", 64, 16, 16), ("bf16", 128, 20, 48), ("f16", 256, 7, 4096)])
def test_pages_further_apart_than_they_are_long(dev, ref, kind, dim, page, extra):
    _case("page stride", kind, dim, page, extra)
    full = [150, 33, 0]
    c = ref.Cache(np.random.default_rng(44), 3, 1 + 150 // page, 2, page, dim, full, extra=extra)
    Attend(dev, ref, c, kind, 6, [100, 0, 0], [50, 33, 0]).check(ref)


# ---- scores of any size ------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,far", [(64, 16, False), (128, 10, False), (256, 32, False), (64, 32, True), (128, 16, True)])
@pytest.mark.parametrize("sign", [1, -1])
def test_tokens_scores_far_beyond_24_bits(dev, ref, kind, dim, page, far, sign):
    """Scores of 2^12 to 2^60, exact in fp32 (one value of q counts, a power of two): the rows of the
    largest score share a token's output, the others are too far below it."""
    _case("tokens scores", kind, dim, page, far, sign)
    rng = np.random.default_rng(45)
    n, new = 310, 49
    c = ref.Cache(rng, 1, -(-n // page), 2, page, dim, [n])
    c.code["k"][..., 0] = rng.integers(0x30, 0x7F, c.code["k"].shape[:3])  # 0.5 to 448
    for j in range(c.width):
        c.scale["k"][c.table[0, j]] = 2.0 ** (20 - (int(rng.integers(0, 30)) if far else j % 2))
    q = np.zeros((new, 4, dim))
    q[:, :, 0] = sign * 2.0 ** (np.arange(new)[:, None] - 16)
    if kind == "f16":
        q = np.clip(q, -2.0 ** 15, 2.0 ** 15)
    a = Attend(dev, ref, c, kind, 4, [n - new], [new], scale=1.0, q=q)
    got, want = a.run(), ref.attend64(c, a.q, a.first, a.length, a.scale)
    _check_each(a, got, want, range(new), 4 * TOL[kind])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 10), (256, 1)])
def test_tokens_large_scores_on_pages_of_powers_far_apart(dev, ref, kind, dim, page):
    """V's powers count whatever the scores' size is (they are a part of the exponent in which the
    scores are)."""
    _case("tokens scores, powers", kind, dim, page)
    rng = np.random.default_rng(51)
    n, new = 150, 60
    c = ref.Cache(rng, 1, -(-n // page), 2, page, dim, [n])
    c.code["k"][..., 0] = rng.integers(0x30, 0x7F, c.code["k"].shape[:3])
    _powers(c, 0, "k", [20] * c.width)
    _powers(c, 0, "v", [(-20, 3, -9, -1)[j % 4] for j in range(c.width)])
    q = np.zeros((new, 4, dim))
    # (every token another order of the rows: its own window)
    q[:, :, 0] = 2.0 ** (np.arange(new)[:, None] % 30 - 12)
    a = Attend(dev, ref, c, kind, 4, [n - new], [new], scale=1.0, q=q, window=13)
    got, want = a.run(), ref.attend64(c, a.q, a.first, a.length, a.scale, 13)
    _check_each(a, got, want, range(new), 4 * TOL[kind])


# ---- one token ------------------------------------------------------------------------------

def _one(dev, ref, c, kind, heads, lens, window=0, mask=None, scale=None, q=None):
    """out [batch][heads][dim] of the one-token form, q as it took it, and its scale."""
    import paper_2601_07892_amd as sh
    cd, scale = c.to(dev), float(np.float32(c.dim ** -0.5 if scale is None else scale))
    if q is None:
        q = np.random.default_rng(46).standard_normal((c.batch, heads, c.dim)) * 2
    q = torch.from_numpy(q.astype(np.float32)).to(ref.TYPES[kind])
    qd, out, dl = q.to(dev), torch.empty_like(q, device=dev), _i32(lens, dev)
    dm = None if mask is None else torch.from_numpy(mask).to(dev)
    d = sh.sherry_attend_desc()
    d.q, d.out, d.length, d.mask, d.mask_stride = qd.data_ptr(), out.data_ptr(), dl.data_ptr(), ref.at(dm), c.rows
    d.heads, d.type, d.window, d.scale = heads, ref.CODES[kind], window, scale
    n = sh.sherry_cache_attend_workspace(cd, d)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=dev)
    d.workspace, d.workspace_bytes = ws.data_ptr(), n
    sh.sherry_cache_attend(cd, d)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), q.float().numpy(), scale


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,window", [(64, 16, 0), (128, 10, 300), (256, 32, 70), (64, 1, 0)])
def test_one_token_over_pages_of_any_powers(dev, ref, kind, dim, page, window):
    _case("one token, any powers", kind, dim, page, window)
    rng = np.random.default_rng(47)
    lens = [700, 33, 1, 90]
    c = ref.Cache(rng, 4, -(-700 // page), 2, page, dim, lens)
    for b in range(4):
        _powers(c, b, "v", rng.integers(-60 if kind != "f16" else -15, 20 if kind != "f16" else 3, c.width))
        _powers(c, b, "k", rng.integers(-45, -5, c.width))
    mask = (rng.random((4, c.rows)) < 0.8).astype(np.uint8)
    mask[2, 0] = 1
    for m in (None, mask):
        got, q, scale = _one(dev, ref, c, kind, 6, lens, window, m)
        want = ref.attend64(c, q, np.arange(5), np.array(lens) - 1, scale, window, m)
        _check_each(None, got, want, range(4), 4 * TOL[kind])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 10)])
@pytest.mark.parametrize("many", [False, True])
def test_zeros_on_pages_of_large_powers(dev, ref, kind, dim, page, many):
    """A row that is masked has given its page a power that times q's passes fp32; the others are
    zeros of that page, and their scores 0.  One new token, and many."""
    _case("zeros", kind, dim, page, many)
    n = 5 * page + 1
    c = ref.Cache(np.random.default_rng(48), 1, 6, 2, page, dim, [n])
    p = c.table[0, 2]
    c.code["k"][p] &= 0x80
    c.code["k"][p, :, 3] = 0x7E
    c.scale["k"][p] = 2.0 ** 119
    mask = np.ones((1, c.rows), np.uint8)
    mask[0, 2 * page + 3] = 0
    q = np.random.default_rng(49).standard_normal((1, 4, dim)) * 2.0 ** 12
    if many:
        a = Attend(dev, ref, c, kind, 4, [n - 1], [1], mask=mask, scale=2.0 ** -3, q=q)
        got, q, scale = a.run(), a.q, a.scale
    else:
        got, q, scale = _one(dev, ref, c, kind, 4, [n], mask=mask, scale=2.0 ** -3, q=q)
    want = ref.attend64(c, q, np.arange(2), np.array([n - 1]), scale, mask=mask)
    assert np.all(np.isfinite(got))
    # (scores of some 2^14 times 2^-22 of the largest terms, 2^-6 in the exponents)
    assert _rel(got[0], want[0]) <= 2.0 ** -4


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 10), (256, 32)])
@pytest.mark.parametrize("sign", [1, -1])
def test_one_token_scores_far_beyond_24_bits(dev, ref, kind, dim, page, sign):
    """As with many tokens."""
    _case("one token, scores", kind, dim, page, sign)
    rng = np.random.default_rng(50)
    lens = [310 - i for i in range(40)]
    c = ref.Cache(rng, 40, -(-310 // page), 2, page, dim, lens)
    c.code["k"][..., 0] = rng.integers(0x30, 0x7F, c.code["k"].shape[:3])
    for b in range(40):
        _powers(c, b, "k", [20 - j % 2 for j in range(c.width)])
    q = np.zeros((40, 4, dim))
    q[:, :, 0] = sign * 2.0 ** (np.arange(40)[:, None] - 16)
    got, q, scale = _one(dev, ref, c, kind, 4, lens, scale=1.0, q=q)
    want = ref.attend64(c, q, np.arange(41), np.array(lens) - 1, scale)
    _check_each(None, got, want, range(40), 4 * TOL[kind])
