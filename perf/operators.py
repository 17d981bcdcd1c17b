"""Cases of the operators around the ternary products of a served decoder layer.

* ``append``: rotary positions on q and k, k and v stored into a paged cache;
* ``attend``: attention of one new token per sequence over its pages, with or
  without the accumulated attention weights that eviction goes by;
* ``evict``: a cache cut down to a number of rows per sequence and head, by
  accumulated attention weight;
* ``epilogue``: the packed ternary product with bias, activation, gate and
  residual (int8 activations of m tokens, or one fp32 token).

``run`` computes the plain form in elementary torch operations, or, with
``own``, calls the library.
"""
from __future__ import annotations

import math
import random
import zlib

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8}
GROUP = 128  # weights per scale with "group" scales


def listed():
    return [
        # one conversation at LLaMA-3.2-1B's heads, a few hundred tokens in: latency
        dict(name="attend_1seq_300", op="attend", batch=1, heads=32, kv=8, dim=64, page=16, lo=300, hi=300,
             cache="bf16", type="f32", window=0, mask=False, weights=False, lens=1),
        # a served batch at LLaMA-3.2-3B's heads, conversations of every length
        # (one of them empty, one of a single token)
        dict(name="attend_32seq_ragged", op="attend", batch=32, heads=24, kv=8, dim=128, page=64, lo=1, hi=8000,
             cache="f16", type="f32", window=0, mask=False, weights=False, lens=2),
        # few long documents at 8B scale: the largest cache read
        dict(name="attend_4seq_130k", op="attend", batch=4, heads=32, kv=8, dim=128, page=32, lo=130001, hi=130001,
             cache="bf16", type="bf16", window=0, mask=False, weights=False, lens=3),
        # an int8 cache kept bounded: weights accumulated, a window over the
        # positions and a mask of single tokens
        dict(name="attend_16seq_i8_weights", op="attend", batch=16, heads=32, kv=8, dim=128, page=16, lo=2000,
             hi=9000, cache="i8", type="f32", window=6000, mask=True, weights=True, lens=4),
        # the new tokens of a decode batch
        dict(name="append_32tok_decode", op="append", tokens=32, seqs=32, heads=24, kv=8, dim=128, page=16,
             cache="bf16", type="f32", start=777, rot=128, pairs=False),
        # a prompt into an int8 cache
        dict(name="append_2048tok_prompt_i8", op="append", tokens=2048, seqs=3, heads=32, kv=8, dim=64, page=64,
             cache="i8", type="f32", start=0, rot=64, pairs=False),
        # a step past the budget: a page's worth of rows leaves
        dict(name="evict_8seq_2304_2048", op="evict", batch=8, kv=8, dim=64, page=16, lo=2304, hi=2304, keep=2048,
             recent=256, cache="bf16", lens=5),
        # long prompts cut down to what is served on
        dict(name="evict_16seq_16k_4k", op="evict", batch=16, kv=8, dim=128, page=64, lo=1000, hi=16384, keep=4096,
             recent=512, cache="f16", lens=6),
        # decode: the gate projection of LLaMA-3.2-1B, silu(gate) * up
        dict(name="epi_1tok_gate_1b", op="epilogue", m=1, n=8192, k=2048, input="f32", scales="channel",
             act="silu", bias=False, gate=True, residual=False),
        # decode of a small batch: a down projection onto the residual stream
        dict(name="epi_16tok_down_group", op="epilogue", m=16, n=2048, k=8192, input="i8", scales="group",
             act="none", bias=True, gate=False, residual=True),
        # sizes that fill neither tiles nor units
        dict(name="epi_37tok_ragged", op="epilogue", m=37, n=300, k=1204, input="i8", scales="tensor",
             act="gelu", bias=True, gate=False, residual=True),
        # prefill: the gate projection at 8B scale
        dict(name="epi_2048tok_gate_8b", op="epilogue", m=2048, n=14336, k=4096, input="i8", scales="channel",
             act="silu", bias=False, gate=True, residual=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_CACHE = 2.1e9    # bytes of keys and values read by the largest listed attention
MAX_OPS = 2.4e11     # 2 m n k of the largest listed product


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "evict", "epilogue", "epilogue"])
    if op == "epilogue":
        n, k = (_log_int(rng, 64, 3500) * 4 for _ in range(2))
        if rng.random() < 0.6:
            n, k = max(128, n // 128 * 128), max(128, k // 128 * 128)
        m = 1 if rng.random() < 0.3 else _log_int(rng, 1, max(1, min(4096, int(MAX_OPS / (2 * n * k)))))
        act = rng.choice(["none", "relu", "relu2", "silu", "gelu", "gelu_tanh"])
        return dict(op=op, m=m, n=n, k=k, input="f32" if m == 1 and rng.random() < 0.6 else "i8",
                    scales=rng.choice(["tensor", "channel", "group"]), act=act, bias=rng.random() < 0.5,
                    gate=rng.random() < 0.4, residual=rng.random() < 0.5)
    kv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 3, 4, 4, 8])
    dim = rng.choice([64, 64, 128, 128, 128, 80, 256])
    page = rng.choice([16, 16, 32, 64, 128, 20])
    cache = rng.choice(["bf16", "bf16", "f16", "i8"])
    if op == "append":
        return dict(op=op, tokens=_log_int(rng, 1, 4096), seqs=rng.randint(1, 32), heads=kv * group, kv=kv, dim=dim,
                    page=page, cache=cache, type=rng.choice(["f32", "f32", "bf16", "f16"]),
                    start=rng.randint(0, 1000), rot=dim if rng.random() < 0.7 else dim // 2, pairs=rng.random() < 0.3)
    if op == "evict":
        batch = _log_int(rng, 1, 32)
        hi = _log_int(rng, 64, min(32768, int(2 * MAX_CACHE / 8 / (batch * kv * dim))))
        keep = max(1, int(hi * rng.uniform(0.1, 1.0)))
        return dict(op=op, batch=batch, kv=kv, dim=dim, page=page, lo=max(1, int(hi * rng.choice([0.1, 1.0]))), hi=hi,
                    keep=keep, recent=rng.randint(0, keep // 2), cache=rng.choice(["bf16", "f16"]),
                    lens=rng.randint(0, 1 << 30))
    batch = _log_int(rng, 1, 64)
    hi = _log_int(rng, 1, min(131072, int(MAX_CACHE / 4 / (batch * kv * dim))))
    weights = rng.random() < 0.3
    return dict(op=op, batch=batch, heads=kv * group, kv=kv, dim=dim, page=page,
                lo=hi if rng.random() < 0.5 else max(1, hi // 10), hi=hi, cache=cache,
                type=rng.choice(["f32", "f32", "bf16", "f16"]),
                window=rng.randint(1, hi) if rng.random() < 0.3 else 0, mask=rng.random() < 0.2, weights=weights,
                lens=rng.randint(0, 1 << 30))


# ---- inputs -------------------------------------------------------------------

def _gen(seed, *key):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr((int(seed),) + key).encode()) + (int(seed) << 32))
    return g


def _randn(shape, *key):
    return torch.randn(shape, generator=_gen(*key), device="cuda")


def _lengths(c):
    """Rows of each sequence: log-uniform in [lo, hi]; of ragged batches of eight
    and more the second has one row and the third none."""
    r = random.Random(c["lens"])
    lens = [_log_int(r, c["lo"], c["hi"]) for _ in range(c["batch"])]
    lens[0] = c["hi"]
    if c["op"] == "attend" and c["batch"] >= 8 and c["lo"] < c["hi"]:
        lens[1:3] = [1, 0]
    return lens


def _quantize(x):
    """int8 values and fp32 scales of the rows of x: s = absmax / 127, rint(x / s)."""
    s = x.abs().amax(-1, keepdim=True) / torch.full((), 127.0, device=x.device)
    q = torch.where(s == 0, torch.zeros_like(x), torch.round(x / s)).clamp(-127, 127)
    return q.to(torch.int8), s.squeeze(-1)


def _i32(values):
    return torch.as_tensor(values, dtype=torch.int32).cuda()


def _cache(seed, c, batch, width, used):
    """Pools of all pages, filled, and a table of distinct pages in random order."""
    pages = batch * width + 3
    shape = (pages, c["kv"], c["page"], c["dim"])
    s = {}
    for name in "kv":
        if c["cache"] != "i8":
            s[name] = torch.empty(shape, dtype=TYPES[c["cache"]], device="cuda").normal_(generator=_gen(seed, name))
            s[name + "_scale"] = None
        else:
            s[name], s[name + "_scale"] = _quantize(_randn(shape, seed, name))
    s["table"] = torch.randperm(pages, generator=_gen(seed, "table"), device="cuda")[:batch * width] \
        .view(batch, width).to(torch.int32)
    return s


def prepare(case, seed):
    c = case
    s = {"case": c}
    if c["op"] == "epilogue":
        n, k, m = c["n"], c["k"], c["m"]
        codes = torch.randint(0, 32, (n, k // 4), generator=_gen(seed, "codes"), device="cuda", dtype=torch.uint8)
        s["t"], s["w"] = _ternary(codes), _pack(codes)
        groups = -(-k // GROUP)
        shape = {"tensor": (1,), "channel": (n,), "group": (n, groups)}[c["scales"]]
        s["w_scale"] = torch.rand(shape, generator=_gen(seed, "ws"), device="cuda") * 0.04 + 0.01
        s["w_scale_value"] = float(s["w_scale"].flatten()[0])
        x = _randn((m, k), seed, "x")
        s["x"], s["x_scale"] = (x, None) if c["input"] == "f32" else _quantize(x)
        s["bias"] = _randn((n,), seed, "bias") if c["bias"] else None
        s["gate"] = _randn((m, n), seed, "gate") if c["gate"] else None
        s["residual"] = _randn((m, n), seed, "residual") if c["residual"] else None
        s["y"] = torch.empty((m, n), device="cuda")
        return s
    if c["op"] == "append":
        t, b = c["tokens"], c["seqs"]
        per = -(-t // b)
        width = -(-(c["start"] + per) // c["page"])
        s.update(_cache(seed, c, b, width, None))
        i = torch.arange(t)
        s["seq"], s["slot"] = _i32(i % b), _i32(c["start"] + i // b)
        s["pos"] = s["slot"]
        s["q"], s["new_k"], s["new_v"] = (
            _randn((t, h, c["dim"]), seed, name).to(TYPES[c["type"]])
            for name, h in (("q", c["heads"]), ("nk", c["kv"]), ("nv", c["kv"])))
        at = torch.arange(width * c["page"], dtype=torch.float64)[:, None] * \
            500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
        s["cos"], s["sin"] = at.cos().float().cuda(), at.sin().float().cuda()
        s["q_out"] = torch.empty_like(s["q"])
        s["weight"] = torch.rand((b, c["kv"], width * c["page"]), generator=_gen(seed, "w"), device="cuda")
        s["position"] = torch.zeros((b, c["kv"], width * c["page"]), dtype=torch.int32, device="cuda")
        return s
    lens, b = _lengths(c), c["batch"]
    s["length"] = _i32(lens)
    width = max(1, -(-max(lens) // c["page"]))
    rows = width * c["page"]
    s.update(_cache(seed, c, b, width, lens))
    if c["op"] == "attend":
        s["q"] = (_randn((b, c["heads"], c["dim"]), seed, "q") * 2).to(TYPES[c["type"]])
        s["out"] = torch.empty_like(s["q"])
        s["mask"] = (torch.rand((b, rows), generator=_gen(seed, "mask"), device="cuda") < 0.95).to(torch.uint8) \
            if c["mask"] else None
        s["weight"] = torch.zeros((b, c["kv"], rows), device="cuda") if c["weights"] else None
        s["position"] = s["q_pos"] = None
        if c["weights"] and c["window"]:  # rows that earlier evictions left in no order
            s["position"] = torch.rand((b, c["kv"], rows), generator=_gen(seed, "p"), device="cuda") \
                .argsort(-1).to(torch.int32)
            s["q_pos"] = torch.full((b,), rows, dtype=torch.int32, device="cuda")
        return s
    s["weight"] = torch.exp(2 * _randn((b, c["kv"], rows), seed, "w"))
    s["weight"] *= torch.rand(s["weight"].shape, generator=_gen(seed, "z"), device="cuda") < 0.98  # rows just written: 0
    s["position"] = torch.rand((b, c["kv"], rows), generator=_gen(seed, "p"), device="cuda").argsort(-1).to(torch.int32)
    s["recent_from"] = torch.full((b,), rows - c["recent"], dtype=torch.int32, device="cuda")
    s["length_out"] = torch.empty(b, dtype=torch.int32, device="cuda")
    for name, dtype in (("kept", torch.int32), ("weight_out", torch.float32), ("position_out", torch.int32)):
        s[name] = torch.empty((b, c["kv"], c["keep"]), dtype=dtype, device="cuda")
    return s


def _ternary(codes):
    """int8 [n][4 * codes] of 5-bit codes z | s0<<2 | s1<<3 | s2<<4: position z is 0,
    the others' signs in ascending position."""
    code = torch.arange(32)
    z = code & 3
    table = torch.zeros((32, 4), dtype=torch.int8)
    for p in range(4):
        i = p - (p > z).long()
        table[:, p] = torch.where(p == z, 0, 1 - 2 * ((code >> (2 + i)) & 1)).to(torch.int8)
    return table.cuda()[codes.long()].view(codes.shape[0], -1)


def _pack(codes):
    """Codes -> units of 64 rows x 32 codes: 16 bytes of each row, then 4 of each."""
    n, kc = codes.shape
    rows, units = -(-n // 64), -(-kc // 32)
    full = torch.zeros((rows * 64, units * 32), dtype=torch.int64, device=codes.device)
    full[:n, :kc] = codes
    eight = full.view(rows, 64, units, 4, 8)
    bits = sum(eight[..., j] << (5 * j) for j in range(8))
    by = torch.stack([(bits >> (8 * j)) & 255 for j in range(5)], -1).to(torch.uint8)
    by = by.view(rows, 64, units, 20).transpose(1, 2)
    return torch.cat([by[..., :16].reshape(rows, units, 1024), by[..., 16:].reshape(rows, units, 256)], -1) \
        .contiguous().view(-1)


# ---- one pass -----------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "evict": _own_evict, "epilogue": _own_epilogue}[c["op"]](state)
    return {"append": _append, "attend": _attend, "evict": _evict, "epilogue": _epilogue}[c["op"]](state)


def _values(s, name):
    """A pool's values: as stored, or what its int8 rows stand for."""
    return s[name] if s[name + "_scale"] is None else s[name] * s[name + "_scale"].unsqueeze(-1)


def _rotate(x, cos, sin, rot, pairs):
    """x [tokens][heads][dim] in 32 bits, cos and sin [tokens][rot / 2]."""
    cos, sin = cos.unsqueeze(1), sin.unsqueeze(1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((ya, yb), -1).flatten(-2) if pairs else torch.cat((ya, yb), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _append(s):
    c = s["case"]
    seq, slot, pos = s["seq"].long(), s["slot"].long(), s["pos"].long()
    cos, sin = s["cos"][pos], s["sin"][pos]
    s["q_out"] = _rotate(s["q"].float(), cos, sin, c["rot"], c["pairs"]).to(s["q"].dtype)
    page = s["table"][seq, slot // c["page"]].long()[:, None]
    off, head = (slot % c["page"])[:, None], torch.arange(c["kv"], device=seq.device)[None, :]
    new = {"k": _rotate(s["new_k"].float(), cos, sin, c["rot"], c["pairs"]), "v": s["new_v"].float()}
    for name, x in new.items():
        if c["cache"] == "i8":
            x, scale = _quantize(x)
            s[name + "_scale"][page, head, off] = scale
        s[name][page, head, off] = x.to(s[name].dtype)
    s["weight"][seq[:, None], head, slot[:, None]] = 0.0
    s["position"][seq[:, None], head, slot[:, None]] = s["pos"][:, None].expand(-1, c["kv"])
    return [s["q_out"], _values(s, "k"), _values(s, "v"), s["weight"], s["position"]]


def _pages(s, name, c):
    """[batch][kv][rows][dim] in 32 bits of the pages of every sequence."""
    t = s["table"].long()
    x = s[name][t].float()
    if s[name + "_scale"] is not None:
        x = x * s[name + "_scale"][t].unsqueeze(-1)
    return x.transpose(1, 2).reshape(t.shape[0], c["kv"], -1, c["dim"])


def _valid(s, c, rows):
    """[batch][kv][rows]: the slots that the new token attends to."""
    at = torch.arange(rows, device=s["length"].device)
    n = s["length"].long()[:, None, None]
    ok = (at < n).expand(-1, c["kv"], -1)
    if c["window"]:
        if s["position"] is not None:
            ok = ok & (s["position"].long() > s["q_pos"].long()[:, None, None] - c["window"])
        else:
            ok = ok & (at >= n - c["window"])
    if s["mask"] is not None:
        ok = ok & (s["mask"] != 0)[:, None, :]
    return ok


def _attend(s):
    c = s["case"]
    b, group = c["batch"], c["heads"] // c["kv"]
    q = s["q"].float().view(b, c["kv"], group, c["dim"])
    k = _pages(s, "k", c)
    score = torch.matmul(q, k.transpose(-1, -2)) * c["dim"] ** -0.5
    del k
    ok = _valid(s, c, score.shape[-1]).unsqueeze(2)
    score = torch.where(ok, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(ok, torch.exp(score - top), 0.0)
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    out = torch.matmul(p, _pages(s, "v", c)).view(b, c["heads"], c["dim"]).to(s["q"].dtype)
    if s["weight"] is None:
        return [out]
    s["weight"] += p.sum(2)
    return [out, s["weight"]]


def _evict(s):
    c = s["case"]
    b, kv, rows = s["weight"].shape
    at = torch.arange(rows, device=s["weight"].device)
    n = s["length"].long()[:, None, None]
    new = n.clamp(max=c["keep"])
    rank = torch.where(s["position"] >= s["recent_from"][:, None, None], math.inf, s["weight"])
    rank = torch.where(at < n, rank, -1.0)
    order = rank.sort(dim=-1, descending=True, stable=True).indices
    keep = torch.zeros((b, kv, rows), dtype=torch.bool, device=at.device)
    keep.scatter_(-1, order, (at < new).expand(b, kv, -1))
    hole, mover = ~keep & (at < new), keep & (at >= new)
    source = torch.full((b, kv, rows + 1), -1, dtype=torch.int64, device=at.device)
    place = torch.where(mover, mover.cumsum(-1) - 1, rows)
    source.scatter_(-1, place, at.expand(b, kv, -1))
    kept = torch.where(hole, source.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), at)
    kept = torch.where(at < new, kept, -1)[..., :c["keep"]]
    if rows < c["keep"]:
        kept = torch.nn.functional.pad(kept, (0, c["keep"] - rows), value=-1)
    some, live = kept.clamp(min=0), kept >= 0
    weight = torch.where(live, s["weight"].gather(-1, some), 0.0)
    position = torch.where(live, s["position"].gather(-1, some), 0)
    # each of the first rows from where it is kept (those past the new length
    # from where they are)
    j = at[:c["keep"]].expand(b, kv, -1)
    r = torch.where(live, kept, -1)[..., :rows]
    r = torch.where(r >= 0, r, j)
    i, h = torch.arange(b, device=at.device)[:, None, None], torch.arange(kv, device=at.device)[None, :, None]
    table = s["table"].long()
    to, source = table[i, j // c["page"]], table[i, r // c["page"]]
    for name in "kv":
        s[name][to, h, j % c["page"]] = s[name][source, h, r % c["page"]]
    return [new.flatten().to(torch.int32), kept.to(torch.int32), weight, position, s["k"], s["v"]]


def _act(x, act):
    if act == "relu":
        return x.clamp(min=0)
    if act == "relu2":
        return x.clamp(min=0).square()
    if act == "silu":
        return x / (1 + torch.exp(-x))
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _epilogue(s):
    c = s["case"]
    x, sx = (s["x"], s["x_scale"]) if c["input"] == "i8" else _quantize(s["x"])
    x, t = x.float(), s["t"].float()
    if c["scales"] == "group":
        t = t * s["w_scale"].repeat_interleave(GROUP, 1)[:, :c["k"]]
        y = torch.matmul(x, t.t()) * sx[:, None]
    else:
        y = torch.matmul(x, t.t()) * (sx[:, None] * s["w_scale"])
    if s["bias"] is not None:
        y = y + s["bias"]
    y = _act(y, c["act"])
    if s["gate"] is not None:
        y = y * s["gate"]
    if s["residual"] is not None:
        y = y + s["residual"]
    return [y]


# ---- the library's calls --------------------------------------------------------

def _sherry():
    import paper_2601_07892_amd as sh
    return sh


def _at(t):
    return t.data_ptr() if t is not None else None


def _code(sh, name):
    return {"f32": sh.SHERRY_F32, "f16": sh.SHERRY_F16, "bf16": sh.SHERRY_BF16, "i8": sh.SHERRY_I8}[name]


def _kept(s, name, make):
    """Descriptors and workspaces that a program fills once for its buffers."""
    if name not in s:
        s[name] = make()
    return s[name]


def _own_cache(sh, s):
    c = s["case"]
    d = sh.sherry_cache_desc()
    d.k, d.v, d.k_scale, d.v_scale = _at(s["k"]), _at(s["v"]), _at(s["k_scale"]), _at(s["v_scale"])
    d.table, d.type = _at(s["table"]), _code(sh, c["cache"])
    d.pages, d.kv_heads, d.page_size, d.head_dim = s["k"].shape
    d.batch, d.table_width = s["table"].shape
    return d


def _own_append(s):
    sh, c = _sherry(), s["case"]

    def make():
        d = sh.sherry_append_desc()
        d.q, d.k, d.v, d.q_out = _at(s["q"]), _at(s["new_k"]), _at(s["new_v"]), _at(s["q_out"])
        d.seq, d.slot, d.pos = _at(s["seq"]), _at(s["slot"]), _at(s["pos"])
        d.cos, d.sin = _at(s["cos"]), _at(s["sin"])
        d.weight, d.position, d.row_stride = _at(s["weight"]), _at(s["position"]), s["weight"].shape[-1]
        d.tokens, d.heads, d.type = c["tokens"], c["heads"], _code(sh, c["type"])
        d.rope_rows, d.rot_dim = s["cos"].shape[0], c["rot"]
        d.pairing = sh.SHERRY_ROPE_PAIRS if c["pairs"] else sh.SHERRY_ROPE_HALVES
        return _own_cache(sh, s), d

    sh.sherry_cache_append(*_kept(s, "descs", make))
    return [s["q_out"], _values(s, "k"), _values(s, "v"), s["weight"], s["position"]]


def _own_attend(s):
    sh, c = _sherry(), s["case"]

    def make():
        cache, d = _own_cache(sh, s), sh.sherry_attend_desc()
        rows = cache.table_width * cache.page_size
        d.q, d.out, d.length, d.mask = _at(s["q"]), _at(s["out"]), _at(s["length"]), _at(s["mask"])
        d.position, d.q_pos, d.weight = _at(s["position"]), _at(s["q_pos"]), _at(s["weight"])
        d.mask_stride = d.row_stride = rows
        d.heads, d.type, d.window, d.scale = c["heads"], _code(sh, c["type"]), c["window"], c["dim"] ** -0.5
        size = sh.sherry_cache_attend_workspace(cache, d)
        s["workspace"] = torch.zeros(max(size, 16), dtype=torch.uint8, device="cuda")
        d.workspace, d.workspace_bytes = _at(s["workspace"]), size
        return cache, d

    sh.sherry_cache_attend(*_kept(s, "descs", make))
    return [s["out"]] if s["weight"] is None else [s["out"], s["weight"]]


def _own_evict(s):
    sh, c = _sherry(), s["case"]

    def make():
        d = sh.sherry_evict_desc()
        d.length, d.weight, d.position = _at(s["length"]), _at(s["weight"]), _at(s["position"])
        d.recent_from, d.length_out, d.kept = _at(s["recent_from"]), _at(s["length_out"]), _at(s["kept"])
        d.weight_out, d.position_out = _at(s["weight_out"]), _at(s["position_out"])
        d.row_stride, d.out_stride, d.keep = s["weight"].shape[-1], c["keep"], c["keep"]
        return _own_cache(sh, s), d

    sh.sherry_cache_evict(*_kept(s, "descs", make))
    return [s["length_out"], s["kept"], s["weight_out"], s["position_out"], s["k"], s["v"]]


def _own_epilogue(s):
    sh, c = _sherry(), s["case"]

    def make():
        e = sh.sherry_epilogue()
        e.bias, e.gate, e.residual = _at(s["bias"]), _at(s["gate"]), _at(s["residual"])
        e.act = {"none": sh.SHERRY_ACT_NONE, "relu": sh.SHERRY_ACT_RELU, "relu2": sh.SHERRY_ACT_RELU2,
                 "silu": sh.SHERRY_ACT_SILU, "gelu": sh.SHERRY_ACT_GELU, "gelu_tanh": sh.SHERRY_ACT_GELU_TANH}[c["act"]]
        return e

    e = _kept(s, "epilogue", make)
    ws = (s["w_scale_value"], None, None)
    if c["scales"] != "tensor":
        ws = (0.0, s["w_scale"], None) if c["scales"] == "channel" else (0.0, None, s["w_scale"])
    if c["input"] == "f32":
        sh.sherry_gemv_f32_epilogue(s["w"], s["x"], None, *ws, e, s["y"], c["n"], c["k"])
    else:
        sh.sherry_gemm_epilogue(s["w"], s["x"], s["x_scale"], *ws, e, s["y"], c["m"], c["n"], c["k"])
    return [s["y"]]


# ---- what a pass cannot do without ------------------------------------------------

def _size(name):
    return {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}[name]


def work(case):
    c = case
    if c["op"] == "epilogue":
        m, n, k = c["m"], c["n"], c["k"]
        scales = {"tensor": 1, "channel": n, "group": n * -(-k // GROUP)}[c["scales"]]
        x = 4 * m * k if c["input"] == "f32" else m * k + 4 * m
        extra = 4 * n * c["bias"] + 4 * m * n * (c["gate"] + c["residual"])
        return {"bytes": n * k * 5 / 32 + 4 * scales + x + extra + 4 * m * n, "flops": 2 * m * n * k}
    dim, kv = c["dim"], c["kv"]
    row = dim * _size(c["cache"]) + (4 if c["cache"] == "i8" else 0)
    if c["op"] == "append":
        t, e = c["tokens"], _size(c["type"])
        return {"bytes": t * ((2 * c["heads"] + 2 * kv) * dim * e + 2 * kv * row + 4 * c["rot"] + 12 + 8 * kv),
                "flops": 3 * t * (c["heads"] + kv) * c["rot"]}
    lens = _lengths(c)
    if c["op"] == "attend":
        full = -(-max(lens) // c["page"]) * c["page"]
        rows, extra = 0.0, sum(lens) * c["mask"]
        for n in lens:  # rows that the token attends to
            if c["window"] and c["weights"]:  # positions in no order
                extra += 4 * n * kv
                n *= min(1.0, c["window"] / full)
            elif c["window"]:
                n = min(n, c["window"])
            rows += n * 0.95 if c["mask"] else n
        extra += 8 * rows * kv * c["weights"]
        return {"bytes": 2 * rows * kv * row + extra + 2 * c["batch"] * c["heads"] * dim * _size(c["type"]),
                "flops": 4 * rows * c["heads"] * dim}
    kept = [min(n, c["keep"]) for n in lens]
    moved = [min(k, n - k) * k // n for n, k in zip(lens, kept)]  # of evenly spread kept rows, those past the new length
    return {"bytes": kv * (8 * sum(lens) + 12 * sum(kept) + 4 * row * sum(moved)), "flops": 0}


# ---- the same in 64 bits -----------------------------------------------------------

def _quantize64(x):
    s = x.abs().amax(-1, keepdim=True) / 127
    return torch.where(s == 0, 0 * x, torch.round(x / s).clamp(-127, 127) * s)


def exact(case, seed):
    """From the definitions, in 64 bits: loops over sequences, complex rotations."""
    c, s = case, prepare(case, seed)
    f = torch.float64
    if c["op"] == "epilogue":
        x = s["x"].to(f) * s["x_scale"].to(f)[:, None] if c["input"] == "i8" else _quantize64(s["x"].to(f))
        ws = s["w_scale"].to(f)
        if c["scales"] == "group":
            pad = -c["k"] % GROUP
            t = torch.nn.functional.pad(s["t"].to(f), (0, pad)).view(c["n"], -1, GROUP) * ws[..., None]
            t = t.reshape(c["n"], -1)[:, :c["k"]]
        else:
            t = s["t"].to(f) * ws.view(-1, 1)
        z = x @ t.t()
        if c["bias"]:
            z = z + s["bias"].to(f)
        a = {"none": lambda v: v, "relu": torch.relu, "relu2": lambda v: torch.relu(v) ** 2,
             "silu": lambda v: v * torch.sigmoid(v), "gelu": lambda v: v * torch.special.ndtr(v),
             "gelu_tanh": lambda v: v * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3))}[c["act"]](z)
        if c["gate"]:
            a = a * s["gate"].to(f)
        return [a + s["residual"].to(f) if c["residual"] else a]
    dim, kv, page = c["dim"], c["kv"], c["page"]
    k, v = (_values(s, n).to(f) if s[n + "_scale"] is None else s[n].to(f) * s[n + "_scale"].to(f)[..., None] for n in "kv") \
        if c["op"] != "attend" else (None, None)
    if c["op"] == "append":
        turn = torch.complex(s["cos"].to(f), s["sin"].to(f))[s["pos"].long()][:, None]
        half = c["rot"] // 2

        def rotate(x):
            x = x.to(f).clone()
            ia, ib = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["pairs"] else (slice(0, half), slice(half, c["rot"]))
            z = torch.complex(x[..., ia].clone(), x[..., ib].clone()) * turn
            x[..., ia], x[..., ib] = z.real, z.imag
            return x

        seq, slot = s["seq"].long(), s["slot"].long()
        at = s["table"].long()[seq, slot // page]
        for pool, x in ((k, rotate(s["new_k"])), (v, s["new_v"].to(f))):
            x = _quantize64(x) if c["cache"] == "i8" else x
            for h in range(kv):
                pool[at, h, slot % page] = x[:, h]
        for h in range(kv):
            s["weight"][seq, h, slot] = 0
        return [rotate(s["q"]), k, v, s["weight"].to(f), None]
    lens = _lengths(c)
    if c["op"] == "attend":
        out = torch.zeros((c["batch"], c["heads"], dim), dtype=f, device="cuda")
        weight = s["weight"].to(f) if c["weights"] else None
        group = c["heads"] // kv
        for b, n in enumerate(lens):
            if not n:
                continue
            pages = s["table"][b, :-(-n // page)].long()
            for h in range(kv):
                rows = [s[name][pages, h].to(f) * (s[name + "_scale"][pages, h].to(f)[..., None] if c["cache"] == "i8" else 1)
                        for name in "kv"]
                kk, vv = (r.reshape(-1, dim)[:n] for r in rows)
                use = torch.ones(n, dtype=torch.bool, device="cuda")
                if c["window"] and s["position"] is not None:
                    use &= s["position"][b, h, :n] > s["q_pos"][b] - c["window"]
                elif c["window"]:
                    use[:max(0, n - c["window"])] = False
                if c["mask"]:
                    use &= s["mask"][b, :n].bool()
                idx = use.nonzero().flatten()
                if not len(idx):
                    continue
                z = s["q"][b, h * group:(h + 1) * group].to(f) @ kk[idx].t() / math.sqrt(dim)
                p = torch.softmax(z, -1)
                out[b, h * group:(h + 1) * group] = p @ vv[idx]
                if weight is not None:
                    weight[b, h, idx] += p.sum(0)
        return [out] if weight is None else [out, weight]
    weight = torch.zeros((c["batch"], kv, c["keep"]), dtype=f, device="cuda")
    table = s["table"].long()
    for b, n in enumerate(lens):
        m = min(n, c["keep"])
        for h in range(kv):
            w = s["weight"][b, h, :n].to(f)
            w = torch.where(s["position"][b, h, :n] >= s["recent_from"][b], math.inf, w)
            best = torch.argsort(-w, stable=True)[:m].sort().values
            low, high = best[best < m], best[best >= m]
            holes = torch.ones(m, dtype=torch.bool, device="cuda")
            holes[low] = False
            to, src = holes.nonzero().flatten(), torch.arange(m, device="cuda")
            src[to] = high
            weight[b, h, :m] = s["weight"][b, h, src].to(f)
            for pool in (k, v):
                pool[table[b, to // page], h, to % page] = pool[table[b, high // page], h, high % page]
    return [None, None, weight, None, k, v]
