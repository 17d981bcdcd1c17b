"""The decoding example, stage by stage: every stage of a layer against 64 bits
on the device's own inputs to it, so that no int8 rounding that falls the other
way is carried on and amplified.  Tolerances are those of the stages' own
tests: products and sums in fp32 within 1e-5 of the terms' magnitudes, attention
2e-6 of the output's norm (1e-5 of a single sequence's); what is stored, and
which rows an eviction keeps, bit for bit."""
import os

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


@pytest.fixture(scope="module")
def ref():
    import cache_reference
    return cache_reference


def _host(t):
    return t.cpu().numpy()


class Mirror:
    """What a layer's cache has to hold, and the stages' references."""

    def __init__(self, ref, layer):
        c = layer.c
        self.ref, self.layer, self.c, self.dim = ref, layer, c, c.hidden // c.heads
        self.rows = [[[] for _ in range(c.kv)] for _ in range(c.batch)]  # (k, v, position) in 64 bits
        self.weight = np.zeros((c.batch, c.kv, 0))

    def product(self, p, x):
        """The product of fp32 activations x and the bound of its fp32 result."""
        q, s = self.ref.quantize32(x)
        t = p.t.astype(np.float64) * _host(p.scale).astype(np.float64)[:, None]
        a = q.astype(np.float64) * s[:, None]
        return a @ t.T, 1e-5 * (np.abs(a) @ np.abs(t).T) + 1e-12

    def near(self, got, want, bound):
        assert np.all(np.abs(_host(got).astype(np.float64).reshape(want.shape) - want) <= bound)

    def stored(self, x):
        if self.c.cache == "i8":
            q, s = self.ref.quantize32(x)
            return q.astype(np.float64) * s[..., None].astype(np.float64)
        return torch.from_numpy(x).to(self.ref.TYPES[self.c.cache]).double().numpy()

    def step(self, x0, pos):
        c, layer, d = self.c, self.layer, self.dim
        layer.step(c.norm)
        torch.cuda.synchronize()
        # q, k, v; q and k turned
        h = _host(c.norm(x0))
        cos, sin = (np.repeat(_host(t)[pos][None], c.batch, 0) for t in (c.cos, c.sin))
        want, bound = self.product(layer.q, h)
        a, b = (want.reshape(c.batch, c.heads, d)[..., i * (d // 2):(i + 1) * (d // 2)] for i in (0, 1))
        turned = np.concatenate((a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]), -1)
        self.near(layer.yq, turned, 2 * bound.max())
        for p, y in ((layer.k, layer.yk), (layer.v, layer.yv)):
            self.near(y, *self.product(p, h))
        k = self.ref.rotate32(_host(layer.yk).reshape(c.batch, c.kv, d), cos, sin, d, False)
        k, v = self.stored(k), self.stored(_host(layer.yv).reshape(c.batch, c.kv, d))
        for i in range(c.batch):
            for g in range(c.kv):
                self.rows[i][g].append((k[i, g], v[i, g], pos))
        n = len(self.rows[0][0])
        # attention over what has to be in the cache, and its accumulated weights
        q = _host(layer.yq).astype(np.float64).reshape(c.batch, c.kv, -1, d)
        out = np.zeros(q.shape)
        added = np.zeros((c.batch, c.kv, n))
        for i in range(c.batch):
            for g in range(c.kv):
                kk, vv = (np.array([r[j] for r in self.rows[i][g]]) for j in (0, 1))
                s = q[i, g] @ kk.T * float(np.float32(d ** -0.5))
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[i, g], added[i, g] = p @ vv, p.sum(0)
        got = _host(layer.attn).astype(np.float64).reshape(out.shape)
        assert np.linalg.norm(got - out) <= 2e-6 * np.linalg.norm(out)
        for i in range(c.batch):
            assert np.linalg.norm(got[i] - out[i]) <= 1e-5 * np.linalg.norm(out[i])
        before = np.pad(self.weight, ((0, 0), (0, 0), (0, n - self.weight.shape[-1])))
        self.weight = _host(layer.weight[0])[..., :n].astype(np.float64)
        assert np.linalg.norm(self.weight - before - added) <= 1e-5 * np.linalg.norm(before + added)
        assert np.array_equal(_host(layer.position[0])[..., :n],
                              np.array([[[r[2] for r in rows] for rows in s] for s in self.rows]))
        # o onto the residual stream, silu(gate) * up, down onto the residual stream
        y, bound = self.product(layer.o, _host(layer.attn))
        mid, mid_bound = _host(x0).astype(np.float64) + y, bound + 1e-6 * np.abs(y)
        x8, sx = _host(layer.x8).astype(np.float64), _host(layer.sx).astype(np.float64)[:, None]
        h = mid / np.sqrt((mid * mid).mean(-1, keepdims=True) + 1e-5)
        assert np.all(np.abs(x8 * sx - h) <= 0.501 * sx + 1e-4)  # (the norm's input is mid within its bound)
        x = x8 * sx
        t = [p.t.astype(np.float64) * _host(p.scale).astype(np.float64)[:, None] for p in (layer.up, layer.gate)]
        self.near(layer.yup, x @ t[0].T, 1e-5 * (np.abs(x) @ np.abs(t[0]).T))
        z, up = x @ t[1].T, _host(layer.yup).astype(np.float64)
        self.near(layer.yff, z / (1 + np.exp(-z)) * up, 2e-5 * (np.abs(x) @ np.abs(t[1]).T) * np.abs(up) + 1e-9)
        y, bound = self.product(layer.down, _host(layer.yff))
        self.near(c.x, mid + y, mid_bound + bound + 1e-6 * (np.abs(mid) + np.abs(y)))

    def evict(self, keep, recent_from):
        """By the weights that the device has accumulated."""
        c, n = self.c, len(self.rows[0][0])
        w = self.weight.astype(np.float32)
        weight = np.zeros((c.batch, c.kv, keep))
        for i in range(c.batch):
            for g in range(c.kv):
                rows = self.rows[i][g]
                plan = self.ref.evict_plan(w[i, g], np.array([r[2] for r in rows]), recent_from, n, keep)
                self.rows[i][g] = [rows[j] for j in plan]
                weight[i, g] = self.weight[i, g, plan]
        self.weight = weight


@pytest.mark.parametrize("cache,kv", [("bf16", 2), ("f16", 4), ("i8", 1)])
def test_decode_stages(decode, ref, cache, kv):
    dev = torch.device("cuda:0")
    steps, keep, page, recent = 44, 24, 8, 6
    d = decode.Decoder(3, 2, 256, 4, kv, 512, keep, recent, page, cache, steps, 50, dev)
    mirrors = [Mirror(ref, layer) for layer in d.layers]
    tokens, rows = torch.tensor([1, 2, 3], device=dev), 0
    for t in range(steps):
        print("[case] example", cache, kv, "step", t, flush=True)
        d.x.copy_(d.embed[tokens])
        for m in mirrors:
            m.step(d.x.clone(), t)
        d.advance()
        rows += 1
        if rows == keep + page:
            for m in mirrors:
                m.evict(keep, t + 1 - recent)
            rows = keep
        assert d.length.tolist() == [rows] * 3
        tokens = (d.norm(d.x) @ d.head.t()).argmax(-1)


def test_example_runs(decode, capsys):
    out = decode.main(["--steps", "60", "--batch", "5", "--budget", "32", "--recent", "8", "--hidden", "512",
                       "--heads", "8", "--kv", "2", "--inter", "1024", "--cache", "i8"])
    assert out.shape == (5, 60)
    assert "rows in the cache" in capsys.readouterr().out
