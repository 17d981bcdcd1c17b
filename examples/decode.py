"""Decodes a batch of sequences through ternary decoder layers with a bounded
key-value cache: every step of a layer between its norms runs in the library.

Per layer and token: the normed activations are quantized (sherry_quantize_act);
q, k and v are one grouped launch (sherry_gemm_batched); sherry_cache_append
turns q and k and stores k and v; sherry_cache_attend attends to the cache and
adds up each row's attention weight; o is a product that adds the residual
stream (sherry_gemm_epilogue, in place); the gate projection's epilogue is
silu(gate) * up, the down projection's the residual again.  When a sequence's
cache passes its budget by a page, sherry_cache_evict cuts it back to the rows
with the largest weights and the most recent ones.

Weights, tokens and embeddings are random: LLaMA-3.2-1B's sizes with --layers
layers by default.  Run:  python examples/decode.py --steps 64 --batch 8
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2601_07892_amd as sh  # noqa: E402
import synth  # noqa: E402


class Product:
    """A packed projection n x k with one weight scale per output channel."""

    def __init__(self, n, k, dev, *key):
        self.n, self.k = n, k
        self.t = synth.ternary_34(n, k, 5, *key)
        self.w = torch.from_numpy(sh.sherry_pack(self.t)).to(dev)
        rng = np.random.default_rng(n + k)
        self.scale = torch.from_numpy((rng.random(n) + 0.5).astype(np.float32) / k ** 0.5).to(dev)


class Layer:
    """One decoder layer with its cache, buffers and descriptors."""

    def __init__(self, c, index, dev):
        self.c = c
        hidden, inter, b, dim = c.hidden, c.inter, c.batch, c.hidden // c.heads
        kv = c.kv * dim
        make = lambda name, n, k: Product(n, k, dev, name, index)  # noqa: E731
        self.q, self.k, self.v = make("q", hidden, hidden), make("k", kv, hidden), make("v", kv, hidden)
        self.o, self.down = make("o", hidden, hidden), make("down", hidden, inter)
        self.gate, self.up = make("gate", inter, hidden), make("up", inter, hidden)
        f = lambda *s: torch.empty(s, device=dev)  # noqa: E731
        i8 = lambda *s: torch.empty(s, dtype=torch.int8, device=dev)  # noqa: E731
        self.x8, self.sx, self.i8, self.si = i8(b, hidden), f(b), i8(b, inter), f(b)
        self.yq, self.yk, self.yv = f(b, hidden), f(b, kv), f(b, kv)
        self.attn, self.yup, self.yff = f(b, hidden), f(b, inter), f(b, inter)
        # q, k and v in one launch
        descs = (sh.sherry_gemm_desc * 3)()
        for d, p, y in zip(descs, (self.q, self.k, self.v), (self.yq, self.yk, self.yv)):
            d.w, d.x, d.x_scale, d.y = p.w.data_ptr(), self.x8.data_ptr(), self.sx.data_ptr(), y.data_ptr()
            d.w_scales, d.n, d.k, d.m = p.scale.data_ptr(), p.n, p.k, b
        self.blocks, self.launch = sh.sherry_gemm_batched_prepare(descs)
        self.descs = torch.from_numpy(sh.descs_to_bytes(descs)).to(dev)
        # the cache: c.budget rows and a page more per sequence
        width = -(-c.rows // c.page)
        pages, rows = b * width, width * c.page
        kind = {"bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8}[c.cache]
        self.pool = [torch.zeros((pages, c.kv, c.page, dim), dtype=kind, device=dev) for _ in range(2)]
        self.scales = [torch.zeros((pages, c.kv, c.page), device=dev) for _ in range(2)] if c.cache == "i8" else None
        self.table = torch.randperm(pages, device=dev).to(torch.int32).view(b, width)
        d = self.cache = sh.sherry_cache_desc()
        d.k, d.v, d.table = self.pool[0].data_ptr(), self.pool[1].data_ptr(), self.table.data_ptr()
        if self.scales:
            d.k_scale, d.v_scale = self.scales[0].data_ptr(), self.scales[1].data_ptr()
        d.type = {"bf16": sh.SHERRY_BF16, "f16": sh.SHERRY_F16, "i8": sh.SHERRY_I8}[c.cache]
        d.pages, d.page_size, d.kv_heads, d.head_dim, d.batch, d.table_width = pages, c.page, c.kv, dim, b, width
        # accumulated weights and positions, and those that an eviction writes
        self.weight = [torch.zeros((b, c.kv, rows), device=dev) for _ in range(2)]
        self.position = [torch.zeros((b, c.kv, rows), dtype=torch.int32, device=dev) for _ in range(2)]
        self.kept = torch.empty((b, c.kv, rows), dtype=torch.int32, device=dev)
        a = self.append = sh.sherry_append_desc()
        a.q, a.q_out, a.k, a.v = self.yq.data_ptr(), self.yq.data_ptr(), self.yk.data_ptr(), self.yv.data_ptr()
        a.seq, a.slot, a.pos = c.seq.data_ptr(), c.length.data_ptr(), c.pos.data_ptr()
        a.cos, a.sin, a.rope_rows, a.rot_dim = c.cos.data_ptr(), c.sin.data_ptr(), c.cos.shape[0], dim
        a.tokens, a.heads, a.type, a.row_stride = b, c.heads, sh.SHERRY_F32, rows
        t = self.attend = sh.sherry_attend_desc()
        t.q, t.out, t.length = self.yq.data_ptr(), self.attn.data_ptr(), c.attended.data_ptr()
        t.heads, t.type, t.scale, t.row_stride = c.heads, sh.SHERRY_F32, dim ** -0.5, rows
        self._weights()
        size = sh.sherry_cache_attend_workspace(d, t)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=dev)
        t.workspace, t.workspace_bytes = self.workspace.data_ptr(), size
        e = self.add = sh.sherry_epilogue()  # onto the residual stream, in place
        e.residual = c.x.data_ptr()
        e = self.swiglu = sh.sherry_epilogue()
        e.act, e.gate = sh.SHERRY_ACT_SILU, self.yup.data_ptr()

    def _weights(self):
        """Points the descriptors at the weights and positions in use (the first of each)."""
        self.append.weight = self.attend.weight = self.weight[0].data_ptr()
        self.append.position = self.position[0].data_ptr()

    def step(self, norm):
        c, b = self.c, self.c.batch
        sh.sherry_quantize_act(norm(c.x), self.x8, self.sx)
        sh.sherry_gemm_batched(self.descs, 3, self.blocks, self.launch)
        sh.sherry_cache_append(self.cache, self.append)
        sh.sherry_cache_attend(self.cache, self.attend)
        sh.sherry_quantize_act(self.attn, self.x8, self.sx)
        sh.sherry_gemm_epilogue(self.o.w, self.x8, self.sx, 0.0, self.o.scale, None, self.add, c.x, b, self.o.n, self.o.k)
        sh.sherry_quantize_act(norm(c.x), self.x8, self.sx)
        sh.sherry_gemm_channel(self.up.w, self.x8, self.sx, self.up.scale, self.yup, None, b, self.up.n, self.up.k)
        sh.sherry_gemm_epilogue(self.gate.w, self.x8, self.sx, 0.0, self.gate.scale, None, self.swiglu, self.yff, b,
                                self.gate.n, self.gate.k)
        sh.sherry_quantize_act(self.yff, self.i8, self.si)
        sh.sherry_gemm_epilogue(self.down.w, self.i8, self.si, 0.0, self.down.scale, None, self.add, c.x, b,
                                self.down.n, self.down.k)

    def evict(self, recent_from, length_out):
        c = self.c
        d = sh.sherry_evict_desc()
        d.length, d.weight, d.position = c.length.data_ptr(), self.weight[0].data_ptr(), self.position[0].data_ptr()
        d.recent_from, d.length_out, d.kept = recent_from.data_ptr(), length_out.data_ptr(), self.kept.data_ptr()
        d.weight_out, d.position_out = self.weight[1].data_ptr(), self.position[1].data_ptr()
        d.row_stride = d.out_stride = self.kept.shape[-1]
        d.keep = c.budget
        sh.sherry_cache_evict(self.cache, d)
        self.weight.reverse()
        self.position.reverse()
        self._weights()


class Decoder:
    def __init__(self, batch, layers, hidden, heads, kv, inter, budget, recent, page, cache, steps, vocab, dev):
        self.batch, self.hidden, self.heads, self.kv, self.inter = batch, hidden, heads, kv, inter
        self.budget, self.recent, self.page, self.cache = budget, recent, page, cache
        self.rows = budget + page + 1
        i32 = lambda v: torch.full((batch,), v, dtype=torch.int32, device=dev)  # noqa: E731
        self.seq = torch.arange(batch, dtype=torch.int32, device=dev)
        self.length, self.attended, self.pos, self.length_out = i32(0), i32(1), i32(0), i32(0)
        dim = hidden // heads
        angle = torch.arange(steps, dtype=torch.float64)[:, None] * \
            500000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
        self.cos, self.sin = angle.cos().float().to(dev), angle.sin().float().to(dev)
        self.x = torch.empty((batch, hidden), device=dev)
        g = torch.Generator(device=dev)
        g.manual_seed(3)
        self.embed, self.head = (torch.randn((vocab, hidden), generator=g, device=dev) for _ in range(2))
        self.layers = [Layer(self, i, dev) for i in range(layers)]
        self.rows_used = 0  # the same for every sequence here, so the host knows it

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)

    def step(self, tokens):
        """Logits of one more token per sequence; its cache row is appended."""
        self.x.copy_(self.embed[tokens])
        for layer in self.layers:
            layer.step(self.norm)
        self.advance()
        return self.norm(self.x) @ self.head.t()

    def advance(self):
        """Every sequence is a row longer; past the budget by a page, all are cut."""
        self.length += 1
        self.attended += 1
        self.pos += 1
        self.rows_used += 1
        if self.rows_used >= self.budget + self.page:
            recent_from = self.pos - self.recent
            for layer in self.layers:
                layer.evict(recent_from, self.length_out)
            self.length.copy_(self.length_out)
            self.attended.copy_(self.length_out + 1)
            self.rows_used = self.budget


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("batch", 8), ("layers", 2), ("hidden", 2048), ("heads", 32), ("kv", 8), ("inter", 8192),
                        ("budget", 256), ("recent", 64), ("page", 16), ("steps", 400), ("vocab", 1000)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--cache", choices=("bf16", "f16", "i8"), default="bf16")
    a = ap.parse_args(argv)
    dev = torch.device("cuda:0")
    torch.cuda.set_device(dev)
    d = Decoder(a.batch, a.layers, a.hidden, a.heads, a.kv, a.inter, a.budget, a.recent, a.page, a.cache, a.steps,
                a.vocab, dev)
    tokens = torch.arange(a.batch, device=dev) % a.vocab
    out = []
    for i in range(a.steps):
        if i == a.steps // 8:  # (the first steps load the kernels)
            torch.cuda.synchronize()
            t = time.perf_counter()
        tokens = d.step(tokens).argmax(-1)
        out.append(tokens)
    torch.cuda.synchronize()
    t = (time.perf_counter() - t) / (a.steps - a.steps // 8)
    print("%d steps of %d sequences, %d layers: %.1f us a step; rows in the cache: %s" % (
        a.steps, a.batch, a.layers, t * 1e6, d.length.tolist()))
    print("first sequence:", [int(v[0]) for v in out[:16]], "...")
    return torch.stack(out, 1)


if __name__ == "__main__":
    main()
