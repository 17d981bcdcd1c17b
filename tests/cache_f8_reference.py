"""Plain references of the e4m3 cache and of the pages that sequences share, from
their definitions: codes as a table of values, attention in 64 bits, tables and pages
by loops over their entries."""
import numpy as np
import torch

import paper_2601_07892_amd as sh

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"bf16": sh.SHERRY_BF16, "f16": sh.SHERRY_F16, "f32": sh.SHERRY_F32, "i8": sh.SHERRY_I8, "f8": sh.SHERRY_F8}


def at(t):
    return t.data_ptr() if t is not None else None


def _value(code):
    e, m = (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return np.nan
    v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
    return -v if code & 128 else v


VALUES = np.array([_value(c) for c in range(256)])
_POSITIVE = VALUES[:127]                       # 0 .. 448, ascending
_MIDDLE = (_POSITIVE[1:] + _POSITIVE[:-1]) / 2


def encode(x):
    """Codes nearest to x (float64, at most 448 in magnitude), ties to the even code; NaN and infinities: NaN."""
    a = np.abs(x)
    low = np.searchsorted(_MIDDLE, a, side="left")    # ties go down
    high = np.searchsorted(_MIDDLE, a, side="right")  # ties go up
    code = np.where(low % 2 == 0, low, high).astype(np.uint8)
    code = np.where(np.isfinite(x), code, 0x7F)
    return (code | (np.signbit(x) & np.isfinite(x)).astype(np.uint8) << 7).astype(np.uint8)


def power_of(x):
    """Exponent of the page's power for the new values x, as extend takes it."""
    x = np.abs(x[np.isfinite(x)].astype(np.float64))
    top = x.max() if len(x) else 0.0
    e = -100
    while 448.0 * 2.0 ** e < top:
        e += 1
    return e


class Cache:
    """Host copies of an e4m3 cache and, with to(), its device buffers: pages in random
    order, NaN in rows past lens, NaN scales in pages past them."""

    def __init__(self, rng, batch, width, kv, page, dim, lens, extra=0, spread=3):
        self.batch, self.width, self.kv, self.page, self.dim = batch, width, kv, page, dim
        self.rows, self.pages = width * page, batch * width + 2
        self.table = rng.permutation(self.pages)[:batch * width].reshape(batch, width).astype(np.int32)
        self.code, self.scale = {}, {}
        live = np.zeros((self.pages, kv, page), bool)
        for b, n in enumerate(lens):
            for r in range(max(0, min(n, self.rows))):
                live[self.table[b, r // page], :, r % page] = True
        for name in "kv":
            code = encode(np.clip(rng.standard_normal((self.pages, kv, page, dim)) * 40, -448, 448))
            code[~live] = 0x7F
            self.code[name] = code
            # (an exponent alone counts: some mantissas are set)
            s = np.exp2(rng.integers(-5 - spread, -4, (self.pages, kv))).astype(np.float32)
            s = np.where(rng.random(s.shape) < 0.3, s * np.float32(1.75), s)
            self.scale[name] = np.where(live.any(-1), s, np.float32(np.nan)).astype(np.float32)
        self.stride = kv * page * dim + extra

    def power(self, name):
        """What codes are multiplied by, [pages][kv]."""
        bits = self.scale[name].view(np.uint32) >> 23 & 0xFF
        return np.exp2(np.clip(bits, 1, 254).astype(np.float64) - 127)

    def to(self, dev):
        self.d, self.ds = {}, {}
        for name in "kv":
            full = np.full((self.pages, self.stride), 0x11, np.uint8)
            full[:, :self.kv * self.page * self.dim] = self.code[name].reshape(self.pages, -1)
            self.d[name] = torch.from_numpy(full).to(dev)
            self.ds[name] = torch.from_numpy(self.scale[name]).to(dev)
        self.dt = torch.from_numpy(self.table).to(dev)
        c = sh.sherry_cache_desc()
        c.k, c.v, c.k_scale, c.v_scale = at(self.d["k"]), at(self.d["v"]), at(self.ds["k"]), at(self.ds["v"])
        c.table, c.page_stride, c.type = at(self.dt), self.stride, sh.SHERRY_F8
        c.pages, c.page_size, c.kv_heads, c.head_dim = self.pages, self.page, self.kv, self.dim
        c.batch, c.table_width = self.batch, self.width
        return c

    def read(self, name):
        """The device's codes and scales; what lies between pages has to be as it was."""
        full = self.d[name].cpu().numpy()
        whole = self.kv * self.page * self.dim
        assert np.all(full[:, whole:] == 0x11)
        return full[:, :whole].reshape(self.code[name].shape), self.ds[name].cpu().numpy()

    def rows64(self, name, b, h, n):
        """float64 [n][dim] of the first n rows, and which of them there are."""
        pages = self.table[b, :-(-n // self.page)].astype(np.int64)
        there = (pages >= 0) & (pages < self.pages)
        i = np.where(there, pages, 0)
        x = VALUES[self.code[name][i, h]] * self.power(name)[i, h][:, None, None]
        return x.reshape(-1, self.dim)[:n], np.repeat(there, self.page)[:n]


def attend64(c, q, first, length, scale, window=0, mask=None):
    """out [tokens][heads][dim]: tokens of no sequence NaN."""
    tokens, heads, dim = q.shape
    group = heads // c.kv
    out = np.full((tokens, heads, dim), np.nan)
    for b in range(c.batch):
        t0, t1 = int(first[b]), int(first[b + 1])
        base = max(0, min(int(length[b]), c.rows))
        for t in range(t0, t1):
            own = base + t - t0
            n = min(own + 1, c.rows)
            low = max(0, own + 1 - window) if window else 0
            for h in range(c.kv):
                k, there = c.rows64("k", b, h, n)
                v, _ = c.rows64("v", b, h, n)
                use = there & (np.arange(n) >= low)
                if mask is not None:
                    use &= mask[b, :n] != 0
                i = np.flatnonzero(use)
                hs = slice(h * group, (h + 1) * group)
                if not len(i):
                    out[t, hs] = 0
                    continue
                s = scale * (q[t, hs].astype(np.float64) @ k[i].T)
                p = np.exp(s - s.max(-1, keepdims=True))
                out[t, hs] = p @ v[i] / p.sum(-1, keepdims=True)
    return out


def extend_plain(c, new, first, length, cos, sin, rot, pairs, pos=None):
    """Codes and scales of K and V after the new rows (fp32 [tokens][kv][dim], k turned
    already), by loops over pages."""
    from cache_reference import rotate32
    tokens = len(new["k"])
    row = np.full(tokens, -1, np.int64)
    seq = np.full(tokens, -1, np.int64)
    for b in range(c.batch):
        for i, t in enumerate(range(int(first[b]), int(first[b + 1]))):
            r = max(0, min(int(length[b]), c.rows)) + i
            if r < c.rows and 0 <= c.table[b, r // c.page] < c.pages:
                seq[t], row[t] = b, r
    where = row if pos is None else np.asarray(pos, np.int64)
    if cos is not None:
        bad = (where < 0) | (where >= len(cos))
        seq[bad] = -1
        w = np.where(bad, 0, where)
        turned = rotate32(new["k"], cos[w], sin[w], rot, pairs)
    else:
        turned = new["k"]
    code = {n: c.code[n].copy() for n in "kv"}
    scale = {n: c.scale[n].copy() for n in "kv"}
    for b in range(c.batch):
        n = max(0, min(int(length[b]), c.rows))
        # (the rows that the call reaches, tokens left out among them)
        reach = range(n, min(n + int(first[b + 1]) - int(first[b]), c.rows))
        for j in sorted({r // c.page for r in reach}):
            p = c.table[b, j]
            if not 0 <= p < c.pages:
                continue
            mine = np.flatnonzero((seq == b) & (row // c.page == j))
            covered = np.array([r % c.page for r in reach if r // c.page == j])
            for name, x in (("k", turned), ("v", new["v"])):
                for h in range(c.kv):
                    e = power_of(x[mine, h])
                    if j * c.page < n:
                        old = float(np.log2(c.power(name)[p, h]))
                        others = np.setdiff1d(np.arange(c.page), covered)
                        if e > old:
                            y = VALUES[code[name][p, h, others]] * 2.0 ** (old - e)
                            keep = code[name][p, h, others]
                            code[name][p, h, others] = np.where(np.isnan(y), keep, encode(y))
                        e = max(e, int(old))
                    scale[name][p, h] = 2.0 ** e
                    with np.errstate(over="ignore"):
                        code[name][p, h, row[mine] % c.page] = encode(x[mine, h].astype(np.float64) * 2.0 ** -e)
    return code, scale, seq >= 0, where


def up(n, page):
    return -(-n // page) if n > 0 else 0


def fork_plain(table, length, pages, page, parent=None, add=None, from_row=None):
    """(table_out, length_out, missing, copies [(from, to)]); the first two None when pages are missing."""
    batch, width = table.shape
    rows = width * page
    out = np.full((batch, width), -1, np.int64)
    n_out, mine = np.zeros(batch, np.int64), np.zeros((batch, width), bool)
    for b in range(batch):
        p = b if parent is None else int(parent[b])
        n = max(0, min(int(length[p]), rows)) if 0 <= p < batch else 0
        n_out[b] = n
        for j in range(up(n, page)):
            out[b, j] = table[p, j] if 0 <= table[p, j] < pages else -1
        total = min(rows, n + (max(0, int(add[b])) if add is not None else 0))
        begin = n if from_row is None else max(0, min(int(from_row[b]), n))
        for r in range(begin, total):
            mine[b, r // page] = True
    places = {}
    for b in range(batch):
        for j in range(width):
            if out[b, j] >= 0:
                places.setdefault(int(out[b, j]), []).append((b, j))
    free = [p for p in range(pages) if p not in places]
    need = []
    for b in range(batch):
        for j in range(width):
            if not mine[b, j]:
                continue
            held = places.get(int(out[b, j]), []) if out[b, j] >= 0 else []
            if len(held) == 1 or (held and all(mine[i] for i in held) and held[-1] == (b, j)):
                continue
            need.append((b, j))
    if len(need) > len(free):
        return None, None, len(need) - len(free), []
    copies = []
    for (b, j), p in zip(need, free):
        if out[b, j] >= 0:
            copies.append((int(out[b, j]), p))
        out[b, j] = p
    return out.astype(np.int32), n_out.astype(np.int32), 0, copies


def compact_plain(table, length, pages, page):
    """(table_out, moved, live, copies)."""
    batch, width = table.shape
    held = np.zeros((batch, width), bool)
    for b in range(batch):
        held[b, :up(max(0, min(int(length[b]), width * page)), page)] = True
    held &= (table >= 0) & (table < pages)
    used = sorted({int(p) for p in table[held]})
    live = len(used)
    holes = [p for p in range(live) if p not in set(used)]
    moved = np.full(pages, -1, np.int32)
    copies = []
    for p in used:
        moved[p] = p if p < live else holes[len(copies)]
        if p >= live:
            copies.append((p, int(moved[p])))
    out = np.where(held, moved[np.where(held, table, 0)], -1).astype(np.int32)
    return out, moved, live, copies
