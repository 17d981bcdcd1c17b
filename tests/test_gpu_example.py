"""The decoding example against the same steps in 64 bits (with the int8
activation and cache roundings of the path), with and without eviction."""
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def decode():
    import importlib.util
    spec = importlib.util.spec_from_file_location("decode_example", os.path.join(ROOT, "examples", "decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _quant(x):
    s = np.abs(x).max(-1, keepdims=True).astype(np.float32) / np.float32(127)
    return np.clip(np.rint(x.astype(np.float32) / s), -127, 127).astype(np.float64) * s


def _norm(x):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5)


class Plain:
    """A layer with every row's k and v kept as the cache's type holds them."""

    def __init__(self, layer):
        self.p = {n: layer.__dict__[n].t.astype(np.float64) * layer.__dict__[n].scale.double().cpu().numpy()[:, None]
                  for n in ("q", "k", "v", "o", "gate", "up", "down")}
        c = layer.c
        self.c, self.dim = c, c.hidden // c.heads
        self.k = [[[] for _ in range(c.kv)] for _ in range(c.batch)]
        self.v = [[[] for _ in range(c.kv)] for _ in range(c.batch)]
        self.w = [[[] for _ in range(c.kv)] for _ in range(c.batch)]
        self.pos = [[[] for _ in range(c.kv)] for _ in range(c.batch)]

    def _stored(self, x):
        if self.c.cache == "i8":
            return _quant(x)
        return torch.from_numpy(x.astype(np.float32)).to(
            torch.bfloat16 if self.c.cache == "bf16" else torch.float16).double().numpy()

    def step(self, x, pos, cos, sin):
        c, d = self.c, self.dim
        h = _quant(_norm(x))
        q, k, v = (h @ self.p[n].T for n in "qkv")
        def turn(y):
            y = y.reshape(c.batch, -1, d)
            a, b = y[..., :d // 2], y[..., d // 2:]
            return np.concatenate((a * cos - b * sin, b * cos + a * sin), -1)
        q, k, v = turn(q), self._stored(turn(k)), self._stored(v.reshape(c.batch, -1, d))
        out = np.zeros((c.batch, c.heads, d))
        group = c.heads // c.kv
        for b in range(c.batch):
            for g in range(c.kv):
                for store, row in ((self.k, k[b, g]), (self.v, v[b, g]), (self.w, 0.0), (self.pos, pos)):
                    store[b][g].append(row)
                kk, vv = np.array(self.k[b][g]), np.array(self.v[b][g])
                for i in range(g * group, (g + 1) * group):
                    s = kk @ q[b, i] * d ** -0.5
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[b, i] = p @ vv
                    self.w[b][g] = list(np.array(self.w[b][g]) + p)
        x = x + _quant(out.reshape(c.batch, -1)) @ self.p["o"].T
        h = _quant(_norm(x))
        gate, up = h @ self.p["gate"].T, h @ self.p["up"].T
        return x + _quant(gate / (1 + np.exp(-gate)) * up) @ self.p["down"].T

    def evict(self, keep, recent_from):
        for b in range(self.c.batch):
            for g in range(self.c.kv):
                w, p = np.array(self.w[b][g]), np.array(self.pos[b][g])
                best = sorted(range(len(w)), key=lambda i: (p[i] < recent_from, -w[i], i))[:keep]
                for store in (self.k, self.v, self.w, self.pos):
                    store[b][g] = [store[b][g][i] for i in best]


@pytest.mark.parametrize("cache,kv", [("bf16", 2), ("f16", 4), ("i8", 1)])
def test_decode_matches_plain_layers(decode, cache, kv):
    """The residual stream after every step.  int8 roundings on the way may fall
    either side of a half in 32 and in 64 bits: one step of one of 256 values is
    1 / (127 * 16) = 5e-4 of the vector's norm, and few of them differ."""
    dev = torch.device("cuda:0")
    steps, keep, page = 44, 24, 8
    d = decode.Decoder(3, 2, 256, 4, kv, 512, keep, 6, page, cache, steps, 50, dev)
    plain = [Plain(layer) for layer in d.layers]
    cos, sin = d.cos.double().cpu().numpy(), d.sin.double().cpu().numpy()
    tokens, rows = torch.tensor([1, 2, 3], device=dev), 0
    for t in range(steps):
        x = d.embed[tokens].double().cpu().numpy()
        for p in plain:
            x = p.step(x, t, cos[t], sin[t])
        logits = d.step(tokens)
        got = d.x.double().cpu().numpy()
        assert np.linalg.norm(got - x) <= 5e-3 * np.linalg.norm(x), t
        rows += 1
        if rows == keep + page:
            for p in plain:
                p.evict(keep, t + 1 - 6)
            rows = keep
        assert d.length.tolist() == [rows] * 3
        # (each head's kept rows: the same positions, where no weights are near a tie)
        if t == steps - 1:
            for layer, p in zip(d.layers, plain):
                pos = layer.position[0].cpu().numpy()
                same = [len(set(pos[b, g, :rows]) & set(p.pos[b][g])) for b in range(3) for g in range(kv)]
                assert min(same) >= rows - 1
        tokens = logits.argmax(-1)


def test_example_runs(decode, capsys):
    out = decode.main(["--steps", "60", "--batch", "5", "--budget", "32", "--recent", "8", "--hidden", "512",
                       "--heads", "8", "--kv", "2", "--inter", "1024", "--cache", "i8"])
    assert out.shape == (5, 60)
    assert "rows in the cache" in capsys.readouterr().out
