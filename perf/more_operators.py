"""Cases of a served cache in 8 bits whose pages sequences share.

* ``extend``: the new tokens of a ragged batch (prompts, chunks, single tokens)
  turned by their rotary angles and stored as e4m3 codes, one power of two per
  page and head; rows that a page holds already follow when its power rises;
* ``attend``: attention of one new token per sequence over that cache;
* ``tokens``: attention of many new tokens per sequence over it, causal;
* ``fork``: sequences that go on from others (beams, parallel samples), with
  pages for their new rows and copies of the shared pages that they will write;
* ``compact``: the pages in use moved to the front of the pool.

``run`` computes the plain form in elementary torch operations, or, with
``own``, calls the library.
"""
from __future__ import annotations

import math
import random
import zlib

import torch

own = False

F8 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i8": torch.int8, "f8": F8}
TOP = 448.0         # the largest e4m3 value
LEAST = -100        # the smallest exponent of a page's power of two


def listed():
    return [
        # a decode step of a served batch, one new token each, at LLaMA-3.2-3B's heads
        dict(name="extend_32tok_decode", op="extend", batch=32, lo=1, hi=2000, lo_new=1, hi_new=1, heads=24, kv=8,
             dim=128, page=16, type="f32", rot=128, pairs=False, lens=1),
        # prompts of every length, some of them second chunks that start inside a page
        dict(name="extend_8_prompts", op="extend", batch=8, lo=0, hi=700, lo_new=37, hi_new=2048, heads=32, kv=8,
             dim=64, page=32, type="bf16", rot=64, pairs=False, lens=2),
        # one conversation at LLaMA-3.2-1B's heads, a few hundred tokens in: latency
        dict(name="attend_1seq_300", op="attend", batch=1, heads=32, kv=8, dim=64, page=16, lo=300, hi=300,
             type="f32", window=0, mask=False, lens=3),
        # a served batch, conversations of every length (one empty, one of a single token)
        dict(name="attend_32seq_ragged", op="attend", batch=32, heads=24, kv=8, dim=128, page=64, lo=1, hi=8000,
             type="bf16", window=0, mask=False, lens=4),
        # few long documents at 8B scale: the largest cache read, some tokens masked
        dict(name="attend_4seq_130k", op="attend", batch=4, heads=32, kv=8, dim=128, page=32, lo=130001, hi=130001,
             type="bf16", window=0, mask=True, lens=5),
        # drafts of five tokens to be verified, each on its own conversation
        dict(name="tokens_16seq_verify", op="tokens", batch=16, heads=32, kv=8, dim=64, page=16, lo=1, hi=6000,
             lo_new=5, hi_new=5, type="f32", window=0, mask=False, lens=6),
        # a batch of prompts from nothing, every length, a sliding window
        dict(name="tokens_6_prompts", op="tokens", batch=6, heads=24, kv=8, dim=128, page=64, lo=0, hi=0, lo_new=100,
             hi_new=2500, type="bf16", window=1024, mask=False, lens=7),
        # a chunk of a long document at 8B scale
        dict(name="tokens_chunk_30k", op="tokens", batch=1, heads=32, kv=8, dim=128, page=32, lo=30011, hi=30011,
             lo_new=2048, hi_new=2048, type="bf16", window=0, mask=False, lens=8),
        # a step of beam search: 4 beams each of 8 requests go on from beams of the same request
        dict(name="fork_8x4_beams", op="fork", batch=32, fan=4, lo=100, hi=1500, kv=8, dim=64, page=16, layers=16,
             cache="bf16", share=0.8, whole=False, lens=9),
        # shared prefixes copied to pages of their own, as eviction needs them
        dict(name="fork_12_private", op="fork", batch=12, fan=6, lo=2000, hi=7000, kv=8, dim=128, page=32, layers=4,
             cache="f8", share=0.7, whole=True, lens=10),
        # a small pool with holes
        dict(name="compact_6seq_i8", op="compact", batch=6, lo=20, hi=900, kv=4, dim=80, page=20, layers=2, cache="i8",
             spare=1.7, lens=11),
        # a large pool of which a third is in use, before its rear is given back
        dict(name="compact_32seq_f8", op="compact", batch=32, lo=500, hi=8000, kv=8, dim=128, page=64, layers=4,
             cache="f8", spare=3.0, lens=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_READ = 1.06e9   # bytes of keys and values that the largest listed attention reads
MAX_FLOPS = 1.0e12  # operations of the largest listed chunk
MAX_SCORES = 2.1e9  # its scores
MAX_MOVED = 3.0e8   # bytes that the largest listed copies read


def draw(rng):
    op = rng.choice(["extend", "attend", "attend", "tokens", "tokens", "fork", "compact"])
    kv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 3, 4, 4, 8, 16])
    dim = rng.choice([64, 64, 128, 128, 128, 80, 256])
    page = rng.choice([16, 16, 32, 64, 128, 20])
    kind = rng.choice(["f32", "bf16", "bf16", "f16"])
    lens = rng.randint(0, 1 << 30)
    some = dict(kv=kv, dim=dim, page=page, lens=lens)
    if op == "extend":
        hi_new = 1 if rng.random() < 0.4 else _log_int(rng, 2, 4096)
        batch = _log_int(rng, 1, 64 if hi_new == 1 else max(1, min(32, 8192 // hi_new)))
        return dict(op=op, batch=batch, lo=0, hi=_log_int(rng, 1, 2000), lo_new=max(1, hi_new // 10), hi_new=hi_new,
                    heads=kv * group, type=kind, rot=dim if rng.random() < 0.7 else dim // 2, pairs=rng.random() < 0.3,
                    **some)
    if op == "attend":
        batch = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, min(131072, int(MAX_READ / 2 / (batch * kv * dim))))
        return dict(op=op, batch=batch, heads=kv * group, lo=hi if rng.random() < 0.5 else max(1, hi // 10), hi=hi,
                    type=kind, window=rng.randint(1, hi) if rng.random() < 0.3 else 0, mask=rng.random() < 0.2, **some)
    if op == "tokens":
        batch, hi_new = _log_int(rng, 1, 16), _log_int(rng, 1, 4096)
        most = MAX_SCORES / (batch * hi_new * kv * group)
        most = min(most, MAX_FLOPS / (4 * batch * hi_new * kv * group * dim), 100000)
        while hi_new > most / 2:  # scores that the plain form can hold
            hi_new, most = max(1, hi_new // 2), most * 2
        hi = 0 if rng.random() < 0.3 else _log_int(rng, 1, max(1, int(most) - hi_new))
        return dict(op=op, batch=batch, heads=kv * group, lo=hi // 5, hi=hi, lo_new=max(1, hi_new // 8), hi_new=hi_new,
                    type=kind, window=rng.randint(1, hi + hi_new) if rng.random() < 0.3 else 0,
                    mask=rng.random() < 0.2, **some)
    layers, cache = rng.choice([1, 2, 4, 16]), rng.choice(["bf16", "f16", "i8", "f8", "f8"])
    per = 2 * layers * kv * dim * _size(cache)
    if op == "fork":
        fan, whole = rng.choice([1, 2, 4, 4, 8]), rng.random() < 0.3
        batch = fan * _log_int(rng, 1, 8)
        hi = _log_int(rng, 20, max(20, min(20000, int(MAX_MOVED / (per * batch)))))
        return dict(op=op, batch=batch, fan=fan, lo=max(1, hi // 10), hi=hi, layers=layers, cache=cache,
                    share=rng.random(), whole=whole, **some)
    batch = _log_int(rng, 1, 32)
    hi = _log_int(rng, 20, max(20, min(20000, int(MAX_MOVED / (per * batch)))))
    return dict(op=op, batch=batch, lo=max(1, hi // 10), hi=hi, layers=layers, cache=cache, spare=rng.uniform(1.0, 4.0),
                **some)


# ---- inputs -------------------------------------------------------------------

def _gen(seed, *key):
    g = torch.Generator(device="cuda")
    g.manual_seed(zlib.crc32(repr((int(seed),) + key).encode()) + (int(seed) << 32))
    return g


def _randn(shape, *key):
    return torch.randn(shape, generator=_gen(*key), device="cuda")


def _ragged(c):
    """Rows that each sequence has, and its new tokens (None: attend, fork, compact)."""
    r = random.Random(c["lens"])
    some = lambda lo, hi: _log_int(r, lo + 1, hi + 1) - 1  # noqa: E731
    if c["op"] == "fork":  # the beams of a request are of one length
        lens = [x for _ in range(c["batch"] // c["fan"]) for x in [some(c["lo"], c["hi"])] * c["fan"]]
        return [min(x, c["hi"]) for x in lens], None
    lens = [some(c["lo"], c["hi"]) for _ in range(c["batch"])]
    lens[0] = c["hi"]
    if c["op"] == "attend" and c["batch"] >= 8 and c["lo"] < c["hi"]:
        lens[1:3] = [1, 0]
    if c["op"] in ("attend", "compact"):
        return lens, None
    new = [some(c["lo_new"], c["hi_new"]) for _ in range(c["batch"])]
    new[0] = c["hi_new"]
    if c["batch"] >= 4 and c["lo_new"] < c["hi_new"]:
        new[1:3] = [1, 0]
    return lens, new


def _i32(values):
    return torch.as_tensor(values, dtype=torch.int32).cuda()


def _pool(seed, c, pages, name):
    """Pages as earlier tokens left them: e4m3 codes of rows of normal values, with
    the power of two that their largest asks for."""
    shape = (pages, c["kv"], c["page"], c["dim"])
    x = _randn(shape, seed, name)
    x *= torch.exp2(torch.randint(-1, 3, shape[:2] + (1, 1), generator=_gen(seed, name, "size"), device="cuda"))
    scale = _power(x.abs().amax((2, 3)))
    return (x / scale[..., None, None]).to(F8), scale


def _power(top):
    """The smallest power of two with top <= 448 of it."""
    e = torch.frexp(top / TOP)
    e = torch.where(e.mantissa == 0.5, e.exponent - 1, e.exponent).masked_fill(top == 0, LEAST)
    return torch.ldexp(torch.ones_like(top), e.clamp(min=LEAST))


def _cache(seed, c, batch, width):
    s = {}
    pages = batch * width + 3
    for name in "kv":
        s[name], s[name + "_scale"] = _pool(seed, c, pages, name)
    s["table"] = torch.randperm(pages, generator=_gen(seed, "table"), device="cuda")[:batch * width] \
        .view(batch, width).to(torch.int32)
    return s


def prepare(case, seed):
    c = case
    s = {"case": c}
    lens, new = _ragged(c)
    b = c["batch"]
    if c["op"] in ("fork", "compact"):
        return _prepare_pages(s, c, seed, lens)
    full = [n + m for n, m in zip(lens, new or [0] * b)]
    width = max(1, -(-max(full) // c["page"]))
    rows = width * c["page"]
    s["length"] = _i32(lens)
    s.update(_cache(seed, c, b, width))
    kind = TYPES[c["type"]]
    if c["op"] == "attend":
        s["q"] = (_randn((b, c["heads"], c["dim"]), seed, "q") * 2).to(kind)
    else:
        s["tokens"], s["most"] = sum(new), max(new)
        s["first"] = _i32([sum(new[:i]) for i in range(b + 1)])
        s["q"] = (_randn((s["tokens"], c["heads"], c["dim"]), seed, "q") * 2).to(kind)
    if c["op"] == "extend":
        size = torch.exp2(torch.randint(-1, 3, (s["tokens"], 1, 1), generator=_gen(seed, "size"), device="cuda"))
        for name in ("new_k", "new_v"):
            s[name] = (_randn((s["tokens"], c["kv"], c["dim"]), seed, name) * size).to(kind)
        at = torch.arange(rows, dtype=torch.float64)[:, None] * \
            500000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
        s["cos"], s["sin"] = at.cos().float().cuda(), at.sin().float().cuda()
    else:
        s["mask"] = (torch.rand((b, rows), generator=_gen(seed, "mask"), device="cuda") < 0.95).to(torch.uint8) \
            if c["mask"] else None
    s["out"] = torch.empty_like(s["q"])
    return s


def _family(c, lens):
    """Which sequence each goes on from: one of its own request; the last ended."""
    r = random.Random(c["lens"] + 1)
    parent = [b // c["fan"] * c["fan"] + r.randrange(c["fan"]) for b in range(c["batch"])]
    if c["batch"] >= 8:
        parent[-1] = -1
    return parent


def _shared(c, lens):
    """Pages that every sequence of a request shares."""
    return [int(n // c["page"] * c["share"]) if c["fan"] > 1 else 0 for n in lens]


def _prepare_pages(s, c, seed, lens):
    b, page = c["batch"], c["page"]
    width = -(-max(lens) // page) + 2
    need = [-(-n // page) for n in lens]
    if c["op"] == "fork":
        pages = sum(need) * (2 if c["whole"] else 1) + 3 * b + 5
        s["parent"], s["add"] = _i32(_family(c, lens)), _i32([1 + b % 3 for b in range(b)])
        s["from"] = _i32([0] * b) if c["whole"] else None
    else:
        pages = int(sum(need) * c["spare"]) + 3
    order = torch.randperm(pages, generator=_gen(seed, "table"), device="cuda").tolist()
    table = torch.full((b, width), -1, dtype=torch.int32)
    shared = _shared(c, lens) if c["op"] == "fork" else [0] * b
    for i, n in enumerate(need):
        head = i // c["fan"] * c["fan"] if c["op"] == "fork" else i
        for j in range(n):
            table[i, j] = table[head, j] if j < shared[i] and head != i else order.pop()
    s["table"], s["length"] = table.cuda(), _i32(lens)
    shape = (c["layers"], pages, c["kv"], page, c["dim"])
    for name in "kv":
        bits = torch.randint(0, 1 << 62, (math.prod(shape) * _size(c["cache"]) // 8,), generator=_gen(seed, name),
                             device="cuda")
        # finite values of any type; of int8 any but -128
        bits = (bits & 0x3777377737773777).view(torch.uint8)
        s[name] = bits.view(TYPES[c["cache"]]).view(shape)
        s[name + "_scale"] = None
        if c["cache"] in ("i8", "f8"):
            s[name + "_scale"] = torch.rand(shape[:4] if c["cache"] == "i8" else shape[:3], device="cuda",
                                            generator=_gen(seed, name, "scale")) + 0.5
    i32 = lambda *n: torch.full(n, -7, dtype=torch.int32, device="cuda")  # noqa: E731
    s["table_out"], s["length_out"], s["missing"] = i32(b, width), i32(b), i32(1)
    s["moved"], s["live"] = i32(pages), i32(1)
    return s


# ---- one pass -----------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"extend": _own_extend, "attend": _own_attend, "tokens": _own_tokens, "fork": _own_fork,
                "compact": _own_compact}[op](state)
    return {"extend": _extend, "attend": _attend, "tokens": _tokens, "fork": _fork, "compact": _compact}[op](state)


def _rotate(x, cos, sin, rot, pairs):
    """x [tokens][heads][dim] in 32 bits, cos and sin [tokens][rot / 2]."""
    cos, sin = cos.unsqueeze(1), sin.unsqueeze(1)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((ya, yb), -1).flatten(-2) if pairs else torch.cat((ya, yb), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _places(s):
    """Each token's sequence and its row there."""
    at = torch.arange(s["tokens"], device=s["first"].device)
    seq = (at[:, None] >= s["first"][None, 1:].long()).sum(1)
    return seq, s["length"].long()[seq] + at - s["first"].long()[seq]


def _extend(s):
    c = s["case"]
    seq, row = _places(s)
    cos, sin = s["cos"][row], s["sin"][row]
    s["out"] = _rotate(s["q"].float(), cos, sin, c["rot"], c["pairs"]).to(s["q"].dtype)
    page = s["table"][seq, row // c["page"]].long()
    new = {"k": _rotate(s["new_k"].float(), cos, sin, c["rot"], c["pairs"]), "v": s["new_v"].float()}
    # pages that begin behind the rows that a sequence has hold nothing yet
    fresh = row // c["page"] * c["page"] >= s["length"].long()[seq]
    for name, x in new.items():
        pool, scale = s[name], s[name + "_scale"]
        old = scale[page].masked_fill(fresh[:, None], 0.0)
        top = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax")
        need = torch.maximum(_power(top)[page], old)
        # rows that are there already, in the page's new power of two
        codes = pool[page].float() * torch.where(old > 0, old / need, 1.0)[..., None, None]
        codes = torch.where(fresh[:, None, None, None], pool[page].float(), codes)
        pool.view(torch.uint8)[page] = codes.to(F8).view(torch.uint8)
        scale[page] = need
        head = torch.arange(c["kv"], device=page.device)[None, :]
        pool.view(torch.uint8)[page[:, None], head, (row % c["page"])[:, None]] = \
            (x / need[..., None]).to(F8).view(torch.uint8)
    return [s["out"], s["k"], s["v"], s["k_scale"], s["v_scale"]]


def _pages(s, name, c):
    """[batch][kv][rows][dim] in 32 bits of the pages of every sequence."""
    t = s["table"].long()
    x = s[name].view(torch.uint8)[t].view(F8).float() * s[name + "_scale"][t][..., None, None]
    return x.transpose(1, 2).reshape(t.shape[0], c["kv"], -1, c["dim"])


def _softmax_pv(score, ok, v):
    """Softmax over what is attended to (nothing: zeros) times v."""
    score = torch.where(ok, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(ok, torch.exp(score - top), 0.0)
    del score
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, 0.0)
    return torch.matmul(p, v)


def _attend(s):
    c = s["case"]
    b, group = c["batch"], c["heads"] // c["kv"]
    q = s["q"].float().view(b, c["kv"], group, c["dim"])
    score = torch.matmul(q, _pages(s, "k", c).transpose(-1, -2)) * c["dim"] ** -0.5
    at = torch.arange(score.shape[-1], device=score.device)
    n = s["length"].long()[:, None]
    ok = at < n
    if c["window"]:
        ok = ok & (at >= n - c["window"])
    if s["mask"] is not None:
        ok = ok & (s["mask"] != 0)
    out = _softmax_pv(score, ok[:, None, None, :], _pages(s, "v", c))
    return [out.view(b, c["heads"], c["dim"]).to(s["q"].dtype)]


def _tokens(s):
    c = s["case"]
    b, m, group = c["batch"], s["most"], c["heads"] // c["kv"]
    seq, row = _places(s)
    place = seq * m + torch.arange(s["tokens"], device=seq.device) - s["first"].long()[seq]
    q = torch.zeros((b * m, c["heads"], c["dim"]), device=seq.device)
    q[place] = s["q"].float()
    q = q.view(b, m, c["kv"], group, c["dim"]).permute(0, 2, 3, 1, 4).reshape(b, c["kv"], group * m, c["dim"])
    score = torch.matmul(q, _pages(s, "k", c).transpose(-1, -2)) * c["dim"] ** -0.5
    at = torch.arange(score.shape[-1], device=seq.device)
    mine = s["length"].long()[:, None, None] + torch.arange(m, device=seq.device)[:, None]  # [b][m][1]
    ok = at <= mine
    if c["window"]:
        ok = ok & (at > mine - c["window"])
    if s["mask"] is not None:
        ok = ok & (s["mask"] != 0)[:, None, :]
    shape = score.shape
    score = score.view(b, c["kv"], group, m, -1)
    ok = ok[:, None, None].expand(score.shape)
    out = _softmax_pv(score.view(shape), ok.reshape(shape), _pages(s, "v", c))
    out = out.view(b, c["kv"], group, m, c["dim"]).permute(0, 3, 1, 2, 4).reshape(b * m, c["heads"], c["dim"])
    return [out[place].to(s["q"].dtype)]


def _values(s):
    """A pool and its scales, as outputs."""
    return [s[n] for n in ("k", "v", "k_scale", "v_scale") if s[n] is not None]


def _copy(s, source, to):
    for x in (s["k"], s["v"], s["k_scale"], s["v_scale"]):
        if x is not None:
            x = x.view(torch.uint8) if x.dtype == F8 else x
            x[:, to] = x[:, source]


def _count(at, where, pages):
    """How often each page stands in at, where `where` holds."""
    at = torch.where(where, at, pages).flatten()
    return torch.zeros(pages + 1, dtype=torch.int64, device=at.device).index_add_(0, at, torch.ones_like(at))[:pages]


def _fork(s):
    c = s["case"]
    b, width = s["table"].shape
    pages, page = s["k"].shape[1], c["page"]
    at = torch.arange(width, device=s["table"].device)
    parent = s["parent"].long()
    some = (parent >= 0) & (parent < b)
    parent = parent.clamp(0, b - 1)
    n = torch.where(some, s["length"].long()[parent], 0)
    t = s["table"].long()[parent]
    t = torch.where((at < -(-n // page)[:, None]) & (t >= 0) & (t < pages), t, -1)
    total = torch.minimum(n + s["add"].long().clamp(min=0), torch.full_like(n, width * page))
    begin = n if s["from"] is None else torch.minimum(s["from"].long().clamp(min=0), n)
    mine = (at >= (begin // page)[:, None]) & (at < -(-total // page)[:, None]) & (total > begin)[:, None]
    held = t >= 0
    count, wanted = _count(t, held, pages), _count(t, held & mine, pages)
    flat = torch.arange(b * width, device=t.device).view(b, width)
    last = torch.full((pages + 1,), -1, dtype=torch.int64, device=t.device) \
        .index_reduce_(0, torch.where(held & mine, t, pages).flatten(), flat.flatten(), "amax")
    i = t.clamp(min=0)
    keeps = (count[i] == 1) | ((count[i] == wanted[i]) & (last[i] == flat))
    need = mine & (~held | ~keeps)
    free = torch.sort((count > 0).long(), stable=True).indices
    missing = (need.sum() - (count == 0).sum()).clamp(min=0)
    got = free[(need.flatten().long().cumsum(0) - 1).clamp(0, pages - 1)].view(b, width)
    ok = missing == 0
    s["table_out"] = torch.where(ok, torch.where(need, got, t).to(torch.int32), s["table_out"])
    s["length_out"] = torch.where(ok, n.to(torch.int32), s["length_out"])
    moved = need & held & ok
    _copy(s, t[moved], got[moved])
    return [s["table_out"], s["length_out"], missing.to(torch.int32).view(1)] + _values(s)


def _compact(s):
    c = s["case"]
    pages, page = s["k"].shape[1], c["page"]
    t = s["table"].long()
    at = torch.arange(t.shape[1], device=t.device)
    held = (at < -(-s["length"].long() // page)[:, None]) & (t >= 0) & (t < pages)
    used = _count(t, held, pages) > 0
    live = used.sum()
    place = torch.arange(pages, device=t.device)
    hole, mover = ~used & (place < live), used & (place >= live)
    holes = torch.sort((~hole).long(), stable=True).indices
    to = torch.where(mover, holes[(mover.long().cumsum(0) - 1).clamp(min=0)], place)
    s["moved"] = torch.where(used, to, -1).to(torch.int32)
    s["table_out"] = torch.where(held, to[t.clamp(min=0)], -1).to(torch.int32)
    _copy(s, place[mover], to[mover])
    return [s["table_out"], s["moved"], live.to(torch.int32).view(1)] + _values(s)


# ---- the library's calls --------------------------------------------------------

def _sherry():
    import paper_2601_07892_amd as sh
    return sh


def _at(t):
    return t.data_ptr() if t is not None else None


def _code(sh, name):
    return {"f32": sh.SHERRY_F32, "f16": sh.SHERRY_F16, "bf16": sh.SHERRY_BF16, "i8": sh.SHERRY_I8,
            "f8": sh.SHERRY_F8}[name]


def _kept(s, name, make):
    """Descriptors and workspaces that a program fills once for its buffers."""
    if name not in s:
        s[name] = make()
    return s[name]


def _workspace(s, d, size):
    s["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    d.workspace, d.workspace_bytes = _at(s["workspace"]), size


def _own_cache(sh, s):
    c = s["case"]
    d = sh.sherry_cache_desc()
    d.k, d.v, d.k_scale, d.v_scale = _at(s["k"]), _at(s["v"]), _at(s["k_scale"]), _at(s["v_scale"])
    d.table, d.type = _at(s["table"]), _code(sh, c.get("cache", "f8"))
    d.pages, d.kv_heads, d.page_size, d.head_dim = s["k"].shape[-4:]
    d.batch, d.table_width = s["table"].shape
    return d


def _own_extend(s):
    sh, c = _sherry(), s["case"]

    def make():
        d = sh.sherry_extend_desc()
        d.q, d.k, d.v, d.q_out = _at(s["q"]), _at(s["new_k"]), _at(s["new_v"]), _at(s["out"])
        d.first, d.length, d.cos, d.sin = _at(s["first"]), _at(s["length"]), _at(s["cos"]), _at(s["sin"])
        d.tokens, d.heads, d.type = s["tokens"], c["heads"], _code(sh, c["type"])
        d.rope_rows, d.rot_dim = s["cos"].shape[0], c["rot"]
        d.pairing = sh.SHERRY_ROPE_PAIRS if c["pairs"] else sh.SHERRY_ROPE_HALVES
        return _own_cache(sh, s), d

    sh.sherry_cache_extend(*_kept(s, "descs", make))
    return [s["out"], s["k"], s["v"], s["k_scale"], s["v_scale"]]


def _own_attend(s):
    sh, c = _sherry(), s["case"]

    def make():
        cache, d = _own_cache(sh, s), sh.sherry_attend_desc()
        d.q, d.out, d.length, d.mask = _at(s["q"]), _at(s["out"]), _at(s["length"]), _at(s["mask"])
        d.mask_stride = cache.table_width * cache.page_size
        d.heads, d.type, d.window, d.scale = c["heads"], _code(sh, c["type"]), c["window"], c["dim"] ** -0.5
        _workspace(s, d, sh.sherry_cache_attend_workspace(cache, d))
        return cache, d

    sh.sherry_cache_attend(*_kept(s, "descs", make))
    return [s["out"]]


def _own_tokens(s):
    sh, c = _sherry(), s["case"]

    def make():
        cache, d = _own_cache(sh, s), sh.sherry_attend_tokens_desc()
        d.q, d.out, d.first, d.length = _at(s["q"]), _at(s["out"]), _at(s["first"]), _at(s["length"])
        d.mask, d.mask_stride = _at(s["mask"]), cache.table_width * cache.page_size
        d.tokens, d.heads, d.type = s["tokens"], c["heads"], _code(sh, c["type"])
        d.window, d.scale = c["window"], c["dim"] ** -0.5
        _workspace(s, d, sh.sherry_cache_attend_tokens_workspace(cache, d))
        return cache, d

    sh.sherry_cache_attend_tokens(*_kept(s, "descs", make))
    return [s["out"]]


def _layers(s, cache, d):
    d.layers, d.layer_stride = s["k"].shape[0], s["k"].stride(0)
    d.scale_layer_stride = s["k_scale"].stride(0) if s["k_scale"] is not None else 0


def _own_fork(s):
    sh = _sherry()

    def make():
        cache, d = _own_cache(sh, s), sh.sherry_fork_desc()
        d.parent, d.length, d.add, d.from_row = _at(s["parent"]), _at(s["length"]), _at(s["add"]), _at(s["from"])
        d.table_out, d.length_out, d.missing = _at(s["table_out"]), _at(s["length_out"]), _at(s["missing"])
        _layers(s, cache, d)
        _workspace(s, d, sh.sherry_cache_fork_workspace(cache, d))
        return cache, d

    sh.sherry_cache_fork(*_kept(s, "descs", make))
    return [s["table_out"], s["length_out"], s["missing"]] + _values(s)


def _own_compact(s):
    sh = _sherry()

    def make():
        cache, d = _own_cache(sh, s), sh.sherry_compact_desc()
        d.length, d.table_out = _at(s["length"]), _at(s["table_out"])
        d.moved, d.live = _at(s["moved"]), _at(s["live"])
        _layers(s, cache, d)
        _workspace(s, d, sh.sherry_cache_compact_workspace(cache, d))
        return cache, d

    sh.sherry_cache_compact(*_kept(s, "descs", make))
    return [s["table_out"], s["moved"], s["live"]] + _values(s)


# ---- what a pass cannot do without ------------------------------------------------

def _size(name):
    return {"f32": 4, "f16": 2, "bf16": 2, "i8": 1, "f8": 1}[name]


def _page_bytes(c):
    """Of a page in every layer, K and V with their scales."""
    scales = {"i8": 4 * c["page"], "f8": 4}.get(c["cache"], 0)
    return 2 * c["layers"] * c["kv"] * (c["page"] * c["dim"] * _size(c["cache"]) + scales)


def _copies(c, lens):
    """Pages that a fork copies: by the definition, over sets of (request, page of it)."""
    page, parent, shared = c["page"], _family(c, lens), _shared(c, lens)
    who = lambda b, j: (b // c["fan"] * c["fan"] if j < shared[b] else b, j)  # noqa: E731
    count, mine = {}, {}
    for b, p in enumerate(parent):
        if p < 0:
            continue
        n, total = lens[p], min(lens[p] + 1 + b % 3, (-(-max(lens) // page) + 2) * page)
        begin = 0 if c["whole"] else n
        for j in range(-(-n // page)):
            key = who(p, j)
            count[key] = count.get(key, 0) + 1
            if begin // page <= j and total > begin:
                mine[key] = mine.get(key, 0) + 1
    return sum(m - (m == count[k]) for k, m in mine.items())


def work(case):
    c = case
    lens, new = _ragged(c)
    b = c["batch"]
    if c["op"] in ("fork", "compact"):
        width = -(-max(lens) // c["page"]) + 2
        need = sum(-(-n // c["page"]) for n in lens)
        if c["op"] == "fork":
            return {"bytes": 2 * _copies(c, lens) * _page_bytes(c) + 8 * b * width, "flops": 0}
        pages = int(need * c["spare"]) + 3
        # of evenly spread pages in use those that lie behind the first `need`
        return {"bytes": 2 * need * (pages - need) / pages * _page_bytes(c) + 8 * b * width + 4 * pages, "flops": 0}
    dim, kv, e = c["dim"], c["kv"], _size(c["type"])
    if c["op"] == "extend":
        t = sum(new)
        touched = sum(-(-(n + m) // c["page"]) - n // c["page"] for n, m in zip(lens, new) if m)
        return {"bytes": t * ((2 * c["heads"] + 2 * kv) * dim * e + 2 * kv * dim + 4 * c["rot"]) + 8 * touched * kv,
                "flops": 3 * t * (c["heads"] + kv) * c["rot"]}
    pairs, rows = 0, 0
    for n, m in zip(lens, new or [1] * b):
        first = n + 1 if c["op"] == "tokens" else n  # rows of the first of them
        if c["window"]:
            grow = max(0, min(m, c["window"] - first + 1))  # tokens whose window is not full
            pairs += grow * first + grow * (grow - 1) // 2 + (m - grow) * min(c["window"], first + m - 1)
            rows += min(first + m - 1, c["window"] + m - 1) if m else 0
        else:
            pairs += m * first + m * (m - 1) // 2
            rows += first + m - 1 if m else 0
    share = 0.95 if c["mask"] else 1.0
    q = sum(new) if new else b
    return {"bytes": 2 * rows * share * kv * dim + rows * c["mask"] + 2 * q * c["heads"] * dim * e,
            "flops": 4 * pairs * share * c["heads"] * dim}


# ---- the same in 64 bits -----------------------------------------------------------

def _e4m3(x):
    """To the nearest value of 3 bits behind the first, at least 2^-9 apart; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    """From the definitions, in 64 bits: loops over sequences, complex rotations."""
    c, s = case, prepare(case, seed)
    lens, new = _ragged(c)
    f, page = torch.float64, c["page"]
    if c["op"] in ("fork", "compact"):
        return None if c["cache"] in ("i8", "f8") else _exact_pages(c, s, lens)
    table = s["table"].long()
    if c["op"] == "extend":
        turn = torch.complex(s["cos"].to(f), s["sin"].to(f))
        half = c["rot"] // 2
        ia, ib = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["pairs"] else \
            (slice(0, half), slice(half, c["rot"]))

        def rotate(x, rows):
            x = x.to(f).clone()
            z = torch.complex(x[..., ia].clone(), x[..., ib].clone()) * turn[rows][:, None]
            x[..., ia], x[..., ib] = z.real, z.imag
            return x

        out, at = torch.zeros(s["q"].shape, dtype=f, device="cuda"), 0
        pool = {n: s[n].to(f) for n in "kv"}
        scale = {n: s[n + "_scale"].to(f) for n in "kv"}
        for b, (n, m) in enumerate(zip(lens, new)):
            now, rows = slice(at, at + m), torch.arange(n, n + m, device="cuda")
            at += m
            out[now] = rotate(s["q"][now], rows)
            for name, x in (("k", rotate(s["new_k"][now], rows)), ("v", s["new_v"][now].to(f))):
                for j in range(n // page, -(-(n + m) // page) if m else 0):
                    r0, r1 = max(n, j * page), min(n + m, (j + 1) * page)
                    p, y = table[b, j], x[r0 - n:r1 - n].transpose(0, 1)
                    power = torch.exp2(torch.ceil(torch.log2(y.abs().amax((1, 2)) / TOP)).clamp(min=LEAST))
                    if j * page < n:
                        old = scale[name][p].clone()
                        power = torch.maximum(power, old)
                        pool[name][p] = _e4m3(pool[name][p] * (old / power)[:, None, None])
                    scale[name][p] = power
                    pool[name][p][:, r0 - j * page:r1 - j * page] = _e4m3(y / power[:, None, None])
        return [out, pool["k"], pool["v"], scale["k"], scale["v"]]
    group, dim = c["heads"] // c["kv"], c["dim"]
    out, at = torch.zeros(s["q"].shape, dtype=f, device="cuda"), 0
    for b, n in enumerate(lens):
        m = new[b] if new else 1
        rows = n + (m if new else 0)
        now, at = slice(at, at + m), at + m
        if not rows or not m:
            continue
        ids = table[b, :-(-rows // page)]
        mine = torch.arange(rows - m, rows, device="cuda")[:, None]
        col = torch.arange(rows, device="cuda")
        use = col <= mine
        if c["window"]:
            use &= col > mine - c["window"]
        if s["mask"] is not None:
            use &= s["mask"][b, :rows].bool()
        for h in range(c["kv"]):
            k, v = ((s[x].view(torch.uint8)[ids, h].view(F8).to(f) * s[x + "_scale"][ids, h].to(f)[:, None, None])
                    .reshape(-1, dim)[:rows] for x in "kv")
            for i in range(h * group, (h + 1) * group):
                z = torch.where(use, s["q"][now, i].to(f) @ k.t() / math.sqrt(dim), -math.inf)
                out[now, i] = torch.nan_to_num(torch.softmax(z, -1)) @ v
    return [out]


def _exact_pages(c, s, lens):
    """The pools alone: whole numbers have no 64-bit value of their own."""
    pages, page, table = s["k"].shape[1], c["page"], s["table"].tolist()
    need = [-(-n // page) for n in lens]
    if c["op"] == "compact":
        used = sorted({p for row, n in zip(table, need) for p in row[:n]})
        live = len(used)
        there = set(used)
        pairs = list(zip((p for p in used if p >= live), (p for p in range(live) if p not in there)))
    else:
        parent, width = _family(c, lens), len(table[0])
        rows = [table[p][:need[p]] if p >= 0 else [] for p in parent]
        refs, pairs = {}, []
        for b, row in enumerate(rows):
            total = min((lens[parent[b]] if parent[b] >= 0 else 0) + 1 + b % 3, width * page)
            begin = 0 if c["whole"] or parent[b] < 0 else lens[parent[b]] // page
            rows[b] = (row, begin, -(-total // page))
            for j, p in enumerate(row):
                refs.setdefault(p, []).append((b, j, begin <= j))
        free = iter([p for p in range(pages) if p not in refs])
        for b, (row, begin, end) in enumerate(rows):
            for j in range(begin, end):
                if j >= len(row):
                    next(free)
                    continue
                held = refs[row[j]]
                if len(held) > 1 and not (all(h[2] for h in held) and (b, j) == held[-1][:2]):
                    pairs.append((row[j], next(free)))
    out = []
    for name in "kv":
        x = s[name].double()
        for source, to in pairs:
            x[:, to] = x[:, source]
        out.append(x)
    return [None, None, None] + out
