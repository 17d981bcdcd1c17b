"""Plain references of the paged cache's operators, in 64 bits (append: in the
fp32 steps that its definition names), and the buffers that their tests share."""
import numpy as np
import torch

import paper_2601_07892_amd as sh

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8}
CODES = {"bf16": sh.SHERRY_BF16, "f16": sh.SHERRY_F16, "f32": sh.SHERRY_F32, "i8": sh.SHERRY_I8}


def at(t):
    return t.data_ptr() if t is not None else None


class Cache:
    """Host copies of a cache and, with dev, its device buffers.  Pages are in
    random order; rows past the lengths hold NaN (int8: any value, NaN scales)."""

    def __init__(self, rng, batch, width, kv, page, dim, kind, lens=None, extra=0, fill="random"):
        self.batch, self.width, self.kv, self.page, self.dim, self.kind = batch, width, kv, page, dim, kind
        self.rows = width * page
        self.pages = batch * width + 2
        self.table = rng.permutation(self.pages)[:batch * width].reshape(batch, width).astype(np.int32)
        whole = kv * page * dim
        self.stride = whole + extra
        self.pool, self.scale = {}, {}
        for name in "kv":
            shape = (self.pages, kv, page, dim)
            if kind == "i8":
                p = torch.from_numpy(rng.integers(-127, 128, shape).astype(np.int8))
                s = (rng.random(shape[:3]) * 0.03 + 0.002).astype(np.float32)
            else:
                p = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TYPES[kind])
                s = None
            if lens is not None:
                live = np.zeros(shape[:3], bool)
                for b, n in enumerate(lens):
                    for r in range(min(n, self.rows)):
                        live[self.table[b, r // page], :, r % page] = True
                if kind == "i8":
                    s[~live] = np.nan
                else:
                    p[torch.from_numpy(~live)] = float("nan")
            full = torch.empty((self.pages, self.stride), dtype=p.dtype)
            full.fill_(1)
            full[:, :whole] = p.reshape(self.pages, -1)
            self.pool[name], self.scale[name] = full, s

    def view(self, name, full=None):
        full = self.pool[name] if full is None else full
        whole = self.kv * self.page * self.dim
        return full[:, :whole].view(self.pages, self.kv, self.page, self.dim)

    def to(self, dev):
        self.d = {n: p.to(dev) for n, p in self.pool.items()}
        self.ds = {n: None if s is None else torch.from_numpy(s).to(dev) for n, s in self.scale.items()}
        self.dt = torch.from_numpy(self.table).to(dev)
        c = sh.sherry_cache_desc()
        c.k, c.v, c.k_scale, c.v_scale = at(self.d["k"]), at(self.d["v"]), at(self.ds["k"]), at(self.ds["v"])
        c.table, c.page_stride, c.type = at(self.dt), self.stride, CODES[self.kind]
        c.pages, c.page_size, c.kv_heads, c.head_dim = self.pages, self.page, self.kv, self.dim
        c.batch, c.table_width = self.batch, self.width
        return c

    def rows64(self, name, b, h, n):
        """float64 [n][dim] of the first n rows (absent pages: NaN)."""
        pages = self.table[b, :-(-n // self.page)].astype(np.int64)
        there = (pages >= 0) & (pages < self.pages)
        at = torch.from_numpy(np.where(there, pages, 0))
        x = self.view(name)[at, h].double().numpy()
        if self.scale[name] is not None:
            x = x * self.scale[name][at.numpy(), h].astype(np.float64)[..., None]
        x[~there] = np.nan
        return x.reshape(-1, self.dim)[:n]


def attend64(c, q, lens, scale, window=0, mask=None, position=None, q_pos=None):
    """out [batch][heads][dim] and the probabilities summed over each group."""
    batch, heads, dim = q.shape
    group = heads // c.kv
    out = np.zeros((batch, heads, dim))
    weight = np.zeros((batch, c.kv, c.rows))
    for b in range(batch):
        n = max(0, min(int(lens[b]), c.rows))
        for h in range(c.kv):
            pages = c.table[b].astype(np.int64)
            use = np.repeat((pages >= 0) & (pages < c.pages), c.page)[:n]
            if window and position is not None:
                use &= position[b, h, :n].astype(np.int64) > int(q_pos[b]) - window
            elif window:
                use[:max(0, n - window)] = False
            if mask is not None:
                use &= mask[b, :n] != 0
            idx = np.flatnonzero(use)
            if not len(idx):
                continue
            k, v = c.rows64("k", b, h, n)[idx], c.rows64("v", b, h, n)[idx]
            s = scale * (q[b, h * group:(h + 1) * group].astype(np.float64) @ k.T)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, h * group:(h + 1) * group] = p @ v
            weight[b, h, idx] = p.sum(0)
    return out, weight


def rotate32(x, cos, sin, rot, pairs):
    """x fp32 [tokens][heads][dim]; cos, sin fp32 [tokens][rot / 2]: each operation rounded."""
    y = x.copy()
    a, b = (np.s_[..., 0:rot:2], np.s_[..., 1:rot:2]) if pairs else (np.s_[..., :rot // 2], np.s_[..., rot // 2:rot])
    c, s = cos[:, None, :], sin[:, None, :]
    y[a] = x[a] * c - x[b] * s
    y[b] = x[b] * c + x[a] * s
    return y


def quantize32(x):
    """int8 rows and fp32 scales (IEEE fp32 steps)."""
    s = (np.abs(x).max(-1, keepdims=True) / np.float32(127)).astype(np.float32)
    with np.errstate(invalid="ignore", divide="ignore"):
        q = np.where(s == 0, np.float32(0), np.clip(np.rint(x / s), -127, 127))
    return q.astype(np.int8), s[..., 0]


def evict_plan(weight, position, recent_from, n, keep):
    """Former slot of each new row of one sequence and head, by the definition:
    recent rows first (lowest slots of them), then by weight, ties to the lowest slot."""
    w = np.where(np.isnan(weight[:n]), -np.inf, weight[:n]).astype(np.float64)
    recent = np.zeros(n, bool) if recent_from is None else position[:n] >= recent_from
    order = sorted(range(n), key=lambda i: (0, 0, i) if recent[i] else (1, -w[i], i))
    best = set(order[:min(n, keep)])
    m = len(best)
    movers = iter(sorted(i for i in best if i >= m))
    return [i if i in best else next(movers) for i in range(m)]
