"""GPU parity of fork and compact, bit for bit against loops over the table."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


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


SIZE = {"bf16": 2, "f16": 2, "i8": 1, "f8": 1}


class Pool:
    """Pools of some layers, with bytes between pages and between layers."""

    def __init__(self, dev, ref, rng, table, pages, kv, page, dim, kind, layers, gap=0):
        import paper_2601_07892_amd as sh
        self.sh, self.layers, self.pages, self.kind = sh, layers, pages, kind
        e = SIZE[kind]
        self.whole, self.stride = kv * page * dim * e, (kv * page * dim + gap) * e
        self.layer = self.stride * pages + gap * e
        self.scales = {"i8": kv * page, "f8": kv}.get(kind, 0)
        self.scale_layer = self.scales * pages + (3 if gap else 0)
        self.host = {n: rng.integers(0, 256, self.layer * layers, dtype=np.uint8) for n in "kv"}
        self.host_scale = {n: rng.random(self.scale_layer * layers, dtype=np.float32) for n in "kv"}
        self.d = {n: torch.from_numpy(x).to(dev) for n, x in self.host.items()}
        self.ds = {n: torch.from_numpy(x).to(dev) for n, x in self.host_scale.items()}
        self.table = torch.from_numpy(table).to(dev)
        c = self.c = sh.sherry_cache_desc()
        c.k, c.v, c.table = self.d["k"].data_ptr(), self.d["v"].data_ptr(), self.table.data_ptr()
        if self.scales:
            c.k_scale, c.v_scale = self.ds["k"].data_ptr(), self.ds["v"].data_ptr()
        c.page_stride, c.type = self.stride // e, ref.CODES[kind]
        c.pages, c.kv_heads, c.page_size, c.head_dim = pages, kv, page, dim
        c.batch, c.table_width = table.shape
        self.layer_stride, self.scale_layer_stride = self.layer // e, self.scale_layer

    def fill(self, d, workspace):
        d.layers, d.layer_stride, d.scale_layer_stride = self.layers, self.layer_stride, self.scale_layer_stride
        n = workspace(self.c, d)
        assert n > 0
        self.ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=self.table.device)
        d.workspace, d.workspace_bytes = self.ws.data_ptr(), n

    def check(self, copies):
        """Every byte is as the copies leave it."""
        assert bool((self.ws[-64:] == 0xFF).all())
        for n in "kv":
            x = self.host[n].copy()
            s = self.host_scale[n].copy()
            for layer in range(self.layers):
                for a, b in copies:
                    i, j = layer * self.layer + a * self.stride, layer * self.layer + b * self.stride
                    x[j:j + self.whole] = self.host[n][i:i + self.whole]
                    i, j = (layer * self.scale_layer + p * self.scales for p in (a, b))
                    s[j:j + self.scales] = self.host_scale[n][i:i + self.scales]
            assert np.array_equal(self.d[n].cpu().numpy(), x)
            assert np.array_equal(self.ds[n].cpu().numpy(), s)


def _i32(a, dev):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(dev)


def _table(rng, batch, width, pages, lens, page, shared):
    """Distinct pages, but for entries that repeat another sequence's."""
    order = list(rng.permutation(pages))
    t = np.full((batch, width), -1, np.int32)
    for b, n in enumerate(lens):
        for j in range(min(width, -(-max(0, n) // page))):
            t[b, j] = t[rng.integers(0, b), j] if b and rng.random() < shared else -1
            if t[b, j] < 0:
                t[b, j] = order.pop()
    return t


class Fork:
    def __init__(self, dev, ref, pool, table, length, parent, add, from_row, in_place=False):
        sh = pool.sh
        self.pool, self.in_place = pool, in_place
        self.args = [_i32(a, dev) for a in (length, parent, add, from_row)]
        self.out = pool.table if in_place else torch.full(table.shape, -9, dtype=torch.int32, device=dev)
        self.n = torch.full((table.shape[0],), -9, dtype=torch.int32, device=dev)
        self.missing = torch.full((1,), -9, dtype=torch.int32, device=dev)
        d = self.d = sh.sherry_fork_desc()
        d.length, d.parent, d.add, d.from_row = (ref.at(a) for a in self.args)
        d.table_out, d.length_out, d.missing = (x.data_ptr() for x in (self.out, self.n, self.missing))
        pool.fill(d, sh.sherry_cache_fork_workspace)

    def check(self, table, want):
        self.pool.sh.sherry_cache_fork(self.pool.c, self.d)
        torch.cuda.synchronize()
        out, n, missing, copies = want
        assert int(self.missing) == missing
        if missing:
            assert bool((self.n == -9).all())
            assert np.array_equal(self.out.cpu().numpy(), table if self.in_place else np.full(table.shape, -9))
        else:
            assert np.array_equal(self.n.cpu().numpy(), n)
            assert np.array_equal(self.out.cpu().numpy(), out)
        self.pool.check(copies)


# batch, width, page, lengths, kv, dim, type, layers, gap, spare pages
FORKS = [
    (1, 1, 16, [0], 1, 16, "bf16", 1, 0, 1),
    (2, 3, 16, [17, 40], 2, 64, "f8", 1, 0, 4),
    (8, 5, 4, [20, 3, 0, 16, 17, 1, 9, 8], 2, 16, "i8", 3, 16, 60),
    (6, 9, 7, [60, 7, 8, 13, 14, 50], 3, 24, "f16", 2, 8, 60),
    (33, 40, 1, [3 * i % 41 for i in range(33)], 1, 8, "bf16", 2, 0, 2000),
    (70, 3, 20, [i % 61 for i in range(70)], 4, 80, "f8", 1, 16, 300),
    (4, 2, 64, [128, 100, 64, 1], 8, 128, "bf16", 2, 0, 20),   # pages of several chunks
]


@pytest.mark.parametrize("case", FORKS, ids=str)
@pytest.mark.parametrize("seed", range(4))
def test_fork(dev, ref, case, seed):
    batch, width, page, lens, kv, dim, kind, layers, gap, spare = case
    _case("fork", case, seed)
    rng = np.random.default_rng(100 + seed)
    pages = sum(-(-n // page) for n in lens) + spare
    table = _table(rng, batch, width, pages, lens, page, 0.5)
    parent = rng.integers(0, batch, batch) if seed else None  # (several times the same)
    if seed == 2:
        parent[rng.integers(0, batch)] = -1
        parent[rng.integers(0, batch)] = batch
    add = rng.integers(-1, 2 * page + 1, batch) if seed != 3 else None
    from_row = rng.integers(-2, max(lens) + 3, batch) if seed > 1 else None
    pool = Pool(dev, ref, rng, table, pages, kv, page, dim, kind, layers, gap)
    f = Fork(dev, ref, pool, table, lens, parent, add, from_row, in_place=seed == 0)
    f.check(table, ref.fork_plain(table, lens, pages, page, parent, add, from_row))


def test_fork_gives_every_sharer_but_one_a_page(dev, ref):
    """All beams go on from one: the last that writes keeps the page, unless one does not write."""
    rng = np.random.default_rng(1)
    table = np.array([[3, 5], [0, 1], [2, 4], [6, 7]], np.int32)
    for add, from_row in (([1, 1, 1, 1], None), ([1, 0, 1, 1], None), ([0, 0, 0, 0], [0, 0, 0, 0]),
                          ([0, 0, 0, 0], [0, 20, 0, 40])):
        pool = Pool(dev, ref, rng, table, 12, 2, 16, 32, "f8", 2)
        f = Fork(dev, ref, pool, table, [20, 9, 9, 9], [0, 0, 0, 0], add, from_row)
        want = ref.fork_plain(table, [20, 9, 9, 9], 12, 16, [0, 0, 0, 0], add, from_row)
        assert want[2] == 0 and len(want[3]) > 0
        f.check(table, want)


def test_fork_without_enough_pages_changes_nothing(dev, ref):
    rng = np.random.default_rng(2)
    table = np.array([[0, 1, -1], [2, 3, -1]], np.int32)
    for in_place in (False, True):
        for pages, missing in ((4, 2), (5, 1), (6, 0)):
            pool = Pool(dev, ref, rng, table, pages, 1, 16, 32, "bf16", 2)
            f = Fork(dev, ref, pool, table, [32, 32], None, [1, 16], None, in_place=in_place)
            want = ref.fork_plain(table, [32, 32], pages, 16, None, [1, 16], None)
            assert want[2] == missing
            f.check(table, want)


def test_fork_of_odd_tables(dev, ref):
    """Pages that do not exist are given out anew where they are written, and a page
    that stands twice in one sequence is shared with itself."""
    rng = np.random.default_rng(3)
    table = np.array([[0, -1, 99, 3], [4, 4, 4, 1], [-5, 2, 2, 0]], np.int32)
    lens = [60, 64, 1000]
    for from_row, add in (([0, 0, 0], None), ([20, 33, 16], [9, 9, 9]), (None, [1, 1, 1]), (None, [2 ** 31 - 1] * 3)):
        pool = Pool(dev, ref, rng, table, 24, 1, 16, 32, "f8", 1)
        f = Fork(dev, ref, pool, table, lens, None, add, from_row)
        f.check(table, ref.fork_plain(table, lens, 24, 16, None, add, from_row))


@pytest.mark.parametrize("case", FORKS, ids=str)
@pytest.mark.parametrize("seed", range(2))
def test_compact(dev, ref, case, seed):
    batch, width, page, lens, kv, dim, kind, layers, gap, spare = case
    _case("compact", case, seed)
    rng = np.random.default_rng(200 + seed)
    pages = sum(-(-n // page) for n in lens) + spare
    table = _table(rng, batch, width, pages, lens, page, 0.3)
    lens = list(lens)
    if seed:  # (some are cut: their pages behind are free)
        lens[0], lens[-1] = lens[0] // 2, -3
        table[batch // 2, 0] = pages + 5
    _compact(dev, ref, rng, table, lens, pages, kv, page, dim, kind, layers, gap, in_place=bool(seed))


def _compact(dev, ref, rng, table, lens, pages, kv, page, dim, kind, layers, gap, in_place=False, moved=True):
    pool = Pool(dev, ref, rng, table, pages, kv, page, dim, kind, layers, gap)
    out = pool.table if in_place else torch.full(table.shape, -9, dtype=torch.int32, device=dev)
    dm, live, dl = (torch.full((n,), -9, dtype=torch.int32, device=dev) for n in (pages, 1, len(lens)))
    dl.copy_(_i32(lens, dev))
    d = pool.sh.sherry_compact_desc()
    d.length, d.table_out, d.live = dl.data_ptr(), out.data_ptr(), live.data_ptr()
    d.moved = dm.data_ptr() if moved else None
    pool.fill(d, pool.sh.sherry_cache_compact_workspace)
    pool.sh.sherry_cache_compact(pool.c, d)
    torch.cuda.synchronize()
    want_table, want_moved, want_live, copies = ref.compact_plain(table, lens, pages, page)
    assert int(live) == want_live
    assert np.array_equal(out.cpu().numpy(), want_table)
    if moved:
        assert np.array_equal(dm.cpu().numpy(), want_moved)
    pool.check(copies)


def test_compact_of_full_empty_and_packed_pools(dev, ref):
    rng = np.random.default_rng(4)
    full = rng.permutation(64).reshape(4, 16).astype(np.int32)
    for lens in ([16 * 4] * 4, [0] * 4, [64, 0, 0, 0], [1, 1, 1, 1]):
        _compact(dev, ref, rng, full, lens, 64, 1, 4, 16, "bf16", 1, 0, moved=lens[1] == 0)
    _compact(dev, ref, rng, np.arange(64, dtype=np.int32).reshape(4, 16), [40, 64, 64, 64], 65, 1, 4, 16, "bf16", 1, 0)
    _compact(dev, ref, rng, np.zeros((1, 1), np.int32), [1], 1, 1, 4, 16, "bf16", 1, 0)


def test_large_pools(dev, ref):
    """More pages than bits that fit on chip, more sequences than places that do."""
    rng = np.random.default_rng(5)
    for pages, batch, width in ((400_000, 3, 500), (330_001, 1500, 7), (120_000, 1100, 3)):
        _case("large", pages, batch, width)
        lens = rng.integers(0, width + 1, batch)
        table = np.full((batch, width), -1, np.int32)
        table[:] = rng.permutation(pages)[:batch * width].reshape(batch, width)
        table[1:, 0] = np.where(rng.random(batch - 1) < 0.5, table[0, 0], table[1:, 0])
        parent, add = rng.integers(0, batch, batch), rng.integers(0, 3, batch)
        pool = Pool(dev, ref, rng, table, pages, 1, 1, 16, "f8", 1)
        f = Fork(dev, ref, pool, table, lens, parent, add, lens // 2)
        f.check(table, ref.fork_plain(table, lens, pages, 1, parent, add, lens // 2))
        _compact(dev, ref, rng, table, lens, pages, 1, 1, 16, "f8", 1, 0)


@pytest.mark.parametrize("pages,batch,width", [(4700, 70, 64), (4200, 64, 64), (9000, 64, 64), (2500, 1, 2100), (3000, 1030, 2)])
def test_fork_of_tables_near_what_a_workgroup_keeps(dev, ref, pages, batch, width):
    """Entries, pages and sequences on both sides of what stays in registers and on chip."""
    _case("fork kept", pages, batch, width)
    rng = np.random.default_rng(7)
    lens = rng.integers(0, width + 1, batch)
    table = rng.permutation(pages)[:batch * width].reshape(batch, width).astype(np.int32)
    table[1:, 0] = np.where(rng.random(batch - 1) < 0.5, table[0, 0], table[1:, 0])
    for in_place in (False, True):
        parent = None if in_place else rng.integers(0, batch, batch)
        add, from_row = rng.integers(0, 3, batch), lens // 3
        want = ref.fork_plain(table, lens, pages, 1, parent, add, from_row)
        pool = Pool(dev, ref, rng, table, pages, 1, 1, 16, "f8", 2)
        Fork(dev, ref, pool, table, lens, parent, add, from_row, in_place=in_place).check(table, want)


def test_beams_fork_extend_attend_compact_in_a_graph(dev, ref):
    """Beams of two requests: fork, new rows, attention of one token, then compact, the steps
    captured and replayed against the same steps run one by one."""
    import paper_2601_07892_amd as sh
    rng = np.random.default_rng(6)
    batch, width, kv, page, dim, heads, pages = 6, 4, 2, 16, 64, 4, 40
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
    pool = {n: torch.zeros((pages, kv, page, dim), dtype=torch.uint8, device=dev) for n in "kv"}
    scale = {n: torch.zeros((pages, kv), device=dev) for n in "kv"}
    tables, length, length_out = [i32(batch, width) for _ in range(3)], i32(batch), i32(batch)
    after, parent, add, missing, live = i32(batch), i32(batch), i32(batch), i32(1), i32(1)
    add.fill_(1)
    first = torch.arange(batch + 1, dtype=torch.int32, device=dev)
    x = {n: torch.zeros((batch, h, dim), device=dev) for n, h in (("q", heads), ("k", kv), ("v", kv))}
    out = torch.zeros((batch, heads, dim), device=dev)

    def cache(table):
        c = sh.sherry_cache_desc()
        c.k, c.v, c.k_scale, c.v_scale = (t.data_ptr() for t in (pool["k"], pool["v"], scale["k"], scale["v"]))
        c.table, c.type, c.pages, c.kv_heads, c.page_size, c.head_dim = table.data_ptr(), sh.SHERRY_F8, pages, kv, page, dim
        c.batch, c.table_width = batch, width
        return c

    c0, c1 = cache(tables[0]), cache(tables[1])
    keep = []

    def workspace(d, n):
        keep.append(torch.empty(n, dtype=torch.uint8, device=dev))
        d.workspace, d.workspace_bytes = keep[-1].data_ptr(), n

    f = sh.sherry_fork_desc()
    f.parent, f.length, f.add, f.table_out = parent.data_ptr(), length.data_ptr(), add.data_ptr(), tables[1].data_ptr()
    f.length_out, f.missing, f.layers = length_out.data_ptr(), missing.data_ptr(), 1
    workspace(f, sh.sherry_cache_fork_workspace(c0, f))
    e = sh.sherry_extend_desc()
    e.q, e.k, e.v, e.q_out = x["q"].data_ptr(), x["k"].data_ptr(), x["v"].data_ptr(), x["q"].data_ptr()
    e.first, e.length, e.tokens, e.heads, e.type = first.data_ptr(), length_out.data_ptr(), batch, heads, sh.SHERRY_F32
    a = sh.sherry_attend_desc()
    a.q, a.out, a.length, a.heads, a.type, a.scale = (x["q"].data_ptr(), out.data_ptr(), after.data_ptr(), heads,
                                                      sh.SHERRY_F32, dim ** -0.5)
    workspace(a, sh.sherry_cache_attend_workspace(c1, a))
    p = sh.sherry_compact_desc()
    p.length, p.table_out, p.live, p.layers = after.data_ptr(), tables[0].data_ptr(), live.data_ptr(), 1
    workspace(p, sh.sherry_cache_compact_workspace(c1, p))

    def step():
        sh.sherry_cache_fork(c0, f)
        sh.sherry_cache_extend(c1, e)
        torch.add(length_out, 1, out=after)
        sh.sherry_cache_attend(c1, a)
        sh.sherry_cache_compact(c1, p)
        length.copy_(after)

    results = []
    for how in ("eager", "graph"):
        rng = np.random.default_rng(7)
        for t in (*pool.values(), *scale.values(), *tables, length):
            t.zero_()
        rows = [[] for _ in range(batch)]  # what each sequence holds
        if how == "graph":
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            for t in (*pool.values(), *scale.values(), *tables, length):
                t.zero_()
        seen = []
        for i in range(40):
            par = rng.integers(0, 3, batch) + 3 * (np.arange(batch) // 3)
            parent.copy_(_i32(par, dev))
            for n in x:
                x[n].copy_(torch.from_numpy(rng.standard_normal(x[n].shape).astype(np.float32)))
            q, k, v = (x[n].double().cpu().numpy() for n in "qkv")
            torch.cuda.synchronize()
            graph.replay() if how == "graph" else step()
            torch.cuda.synchronize()
            assert int(missing) == 0
            rows = [rows[par[b]] + [(k[b], v[b])] for b in range(batch)]
            t = tables[0].cpu().numpy()
            reached = {int(z) for b in range(batch) for z in t[b, :-(-(i + 1) // page)]}
            assert reached == set(range(int(live)))
            got = out.double().cpu().numpy()
            for b in range(batch):
                for h in range(heads):
                    kk = np.array([r[0][h // 2] for r in rows[b]])
                    vv = np.array([r[1][h // 2] for r in rows[b]])
                    s = kk @ q[b, h] * dim ** -0.5
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    # codes are off by 2^-4 of each value at most, twice that after a page's power rose: scores by
                    # 2^-3 |q| . |k|, so weights by a factor exp(2 * that), and values by 2^-3 of theirs
                    slack = np.exp(2 * (2.0 ** -3 * np.abs(kk) @ np.abs(q[b, h]) * dim ** -0.5).max()) - 1
                    assert np.all(np.abs(got[b, h] - w @ vv) <= (2.0 ** -3 + slack * 1.125) * (w @ np.abs(vv)) + 1e-3)
            seen.append([got.copy(), t.copy(), *(z.cpu().numpy() for z in (*pool.values(), *scale.values()))])
        results.append(seen)
    for one, two in zip(*results):
        for y, z in zip(one, two):
            assert np.array_equal(y, z)
