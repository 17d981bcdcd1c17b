"""GPU parity of the products with an epilogue, y = act(p + bias) * gate +
residual, against 64 bits on the oracle's exact int32 sums.

Tolerance, from the fp32 steps (u = 2^-24): p = float(acc) * (sx * sw) is within
2u |p|, the bias sum adds u |z|; an activation with |act'| <= L passes that on
and adds 8u of its own intermediate values (|z|, or z^2 for relu2); the gate, the
residual and their roundings follow.  Per-group scales: p within (G + 4) u of
its terms' magnitudes."""
import sys

import numpy as np
import pytest

import oracle
import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ACTS = ["none", "relu", "relu2", "silu", "gelu", "gelu_tanh"]


@pytest.fixture(scope="module")
def dev():
    d = torch.device("cuda:0")
    torch.cuda.set_device(d)
    return d


def _act(z, act):
    from scipy.special import erf, expit
    if act == "relu":
        return np.maximum(z, 0)
    if act == "relu2":
        return np.maximum(z, 0) ** 2
    if act == "silu":
        return z * expit(z)
    if act == "gelu":
        return 0.5 * z * (1 + erf(z / np.sqrt(2)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    return z


class Problem:
    def __init__(self, dev, m, n, k, scales, f32, seed=1, sw=0.02):
        import paper_2601_07892_amd as sh
        self.sh, self.dev, self.m, self.n, self.k, self.scales, self.f32 = sh, dev, m, n, k, scales, f32
        rng = self.rng = np.random.default_rng(seed * 7919 + m * 31 + n + k)
        t = synth.ternary_34(n, k, 15, "epi", seed)
        x = synth.activations(m, k, 15, "epi", m, seed)
        q, sx, acc, _ = oracle.linear(x, t, 1.0)
        groups = -(-k // 128)
        self.w = torch.from_numpy(sh.sherry_pack(t)).to(dev)
        s = {"tensor": np.float32(sw), "channel": (rng.random(n) * 2 * sw + 1e-3).astype(np.float32),
             "group": (rng.random((n, groups)) * 2 * sw + 1e-3).astype(np.float32)}[scales]
        if scales == "group":
            tp = np.zeros((n, groups * 128), np.float64)
            tp[:, :k] = t
            qp = np.zeros((m, groups * 128), np.float64)
            qp[:, :k] = q
            parts = np.einsum("mgi,ngi->mng", qp.reshape(m, groups, 128), tp.reshape(n, groups, 128), optimize=True)
            terms = parts * s.astype(np.float64)
            self.p = terms.sum(-1) * sx[:, None]
            self.perr = (groups + 4) * U * np.abs(terms).sum(-1) * sx[:, None]
        else:
            self.p = acc.astype(np.float64) * sx.astype(np.float64)[:, None] * np.float64(s)
            self.perr = 2 * U * np.abs(self.p)
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        self.ds = None if scales == "tensor" else up(s)
        self.ws = (float(s), None, None) if scales == "tensor" else \
            (0.0, self.ds, None) if scales == "channel" else (0.0, None, self.ds)
        self.x = up(x) if f32 else up(q)
        self.sx, self.sx_host = up(sx), sx

    def call(self, e, y):
        if self.f32:
            self.sx.fill_(-1)
            self.sh.sherry_gemv_f32_epilogue(self.w, self.x, self.sx, *self.ws, e, y, self.n, self.k)
        else:
            self.sh.sherry_gemm_epilogue(self.w, self.x, self.sx, *self.ws, e, y, self.m, self.n, self.k)
        torch.cuda.synchronize()
        assert np.array_equal(self.sx.cpu().numpy(), self.sx_host)

    def plain(self):
        """The library's product without an epilogue."""
        sh, y = self.sh, torch.empty((self.m, self.n), device=self.dev)
        w, s = self.w, self.ws
        if self.f32:
            a = (w, self.x, None)
            if self.scales == "tensor":
                sh.sherry_gemv_f32(*a, s[0], y, None, self.n, self.k)
            elif self.scales == "channel":
                sh.sherry_gemv_f32_channel(*a, s[1], y, None, self.n, self.k)
            else:
                sh.sherry_gemv_f32_group(*a, s[2], y, None, self.n, self.k)
        else:
            a, kernel = (w, self.x, self.sx), sh.SHERRY_KERNEL_GEMV if self.m <= 4 else sh.SHERRY_KERNEL_SKINNY
            if self.scales == "tensor":
                sh.sherry_gemm_ex(*a, s[0], y, None, self.m, self.n, self.k, kernel)
            elif self.scales == "channel":
                sh.sherry_gemm_channel(*a, s[1], y, None, self.m, self.n, self.k, kernel)
            else:
                sh.sherry_gemm_group(*a, s[2], y, None, self.m, self.n, self.k, kernel)
        torch.cuda.synchronize()
        return y

    def check(self, act, bias, gate, residual, pad=0, offset=0):
        sh, m, n, rng = self.sh, self.m, self.n, self.rng

        def rows(m, wide, on):
            """A host matrix and its device copy: rows of n in `wide`, the rest NaN."""
            if not on:
                return None, None
            a = rng.standard_normal((m, n)).astype(np.float32)
            flat = torch.full((offset + m * wide,), float("nan"))
            flat[offset:].view(m, wide)[:, :n] = torch.from_numpy(a)
            return a.astype(np.float64), flat.to(self.dev)

        e = sh.sherry_epilogue()
        e.act = getattr(sh, "SHERRY_ACT_" + act.upper())
        b, db = rows(1, n, bias)
        g, dg = rows(m, n + pad, gate)
        r, dr = rows(m, n + 2 * pad, residual)
        for name, d in (("bias", db), ("gate", dg), ("residual", dr)):
            setattr(e, name, None if d is None else d.data_ptr() + 4 * offset)
        e.gate_stride, e.residual_stride = (n + pad if pad else 0), (n + 2 * pad if pad else 0)
        flat = torch.full((m * n + 9 + offset,), float("nan"), device=self.dev)
        y = flat[offset:offset + m * n].view(m, n)
        self.call(e, y)
        got = y.double().cpu().numpy()
        assert bool(torch.isnan(flat[:offset]).all()) and bool(torch.isnan(flat[offset + m * n:]).all())
        z = self.p + (b if bias else 0)
        a = _act(z, act)
        slope = 1.2 if act != "relu2" else 2 * np.abs(z)
        own = 8 * U * (z ** 2 if act == "relu2" else np.abs(z)) if act != "none" else 0
        err = slope * (self.perr + U * np.abs(z) * bool(bias)) + own
        if gate:
            a = a * g
            err = err * np.abs(g) + U * np.abs(a)
        if residual:
            a = a + r
            err = err + U * np.abs(a)
        bad = np.abs(got - a) > 1.01 * err + 1e-37
        assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], a[bad][:4])


# every kernel and shape class: VALU GEMV of 1 to 4 tokens, the register-decoded
# kernel's workgroups, sizes that fill neither tiles, units nor pieces
SIZES = [(1, 1, 4), (1, 65, 132), (2, 130, 1028), (3, 64, 512), (4, 300, 260), (5, 1, 4), (33, 66, 68), (16, 300, 2048),
         (70, 130, 1032), (37, 301, 1204), (100, 514, 384), (130, 1030, 256), (300, 330, 644), (257, 258, 12292),
         (513, 2052, 132)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("scales", ["tensor", "channel", "group"])
def test_epilogue(dev, m, n, k, scales):
    print("[case] epilogue", m, n, k, scales, file=sys.stderr, flush=True)
    p = Problem(dev, m, n, k, scales, False)
    for i, (bias, gate, residual) in enumerate([(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 1), (1, 0, 1)]):
        p.check(ACTS[(i + m + n) % 6], bias, gate, residual, pad=(0, 4, 3)[i % 3], offset=(0, 0, 1)[(i + m) % 3])


@pytest.mark.parametrize("n,k", [(1, 4), (65, 132), (300, 2048), (514, 2052), (70, 8196), (130, 16384), (64, 32768)])
@pytest.mark.parametrize("scales", ["tensor", "channel", "group"])
def test_epilogue_one_fp32_token(dev, n, k, scales):
    print("[case] fp32 epilogue", n, k, scales, file=sys.stderr, flush=True)
    p = Problem(dev, 1, n, k, scales, True)
    for i, act in enumerate(ACTS):
        p.check(act, i & 1, i & 2, (i + 1) & 2, pad=i % 3, offset=i % 2)


@pytest.mark.parametrize("m,f32", [(1, True), (3, False), (40, False)])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("sw", [1e-6, 0.02, 3.0])
def test_activations_over_their_range(dev, m, f32, act, sw):
    """Arguments of about 1e-3, 10 and 1e3: where exp, erf and tanh are near 0,
    in their middle and past their ends."""
    Problem(dev, m, 130, 512, "tensor", f32, seed=3, sw=sw).check(act, False, True, False)


@pytest.mark.parametrize("m,n,k", [(1, 300, 260), (4, 64, 512), (40, 130, 644), (130, 1028, 256)])
@pytest.mark.parametrize("scales", ["tensor", "channel", "group"])
def test_no_epilogue_is_the_product(dev, m, n, k, scales):
    for f32 in ([False, True] if m == 1 else [False]):
        p = Problem(dev, m, n, k, scales, f32)
        y = torch.empty((m, n), device=dev)
        p.call(p.sh.sherry_epilogue(), y)
        assert torch.equal(y, p.plain())


@pytest.mark.parametrize("m,n,k", [(1, 300, 260), (4, 67, 512), (40, 130, 644), (130, 1028, 256), (37, 301, 1204)])
def test_residual_or_gate_in_place(dev, m, n, k):
    """y as its own residual, then as its own gate."""
    for f32 in ([False, True] if m == 1 else [False]):
        p = Problem(dev, m, n, k, "channel", f32)
        start = torch.randn((m, n), device=dev)
        y, apart = start.clone(), torch.empty_like(start)
        for name in ("residual", "gate"):
            e = p.sh.sherry_epilogue()
            e.act = p.sh.SHERRY_ACT_SILU
            setattr(e, name, start.data_ptr())
            p.call(e, apart)
            y.copy_(start)
            setattr(e, name, y.data_ptr())
            p.call(e, y)
            assert torch.equal(y, apart)


def test_infinities_and_nan(dev):
    """What a gate, bias or residual holds reaches its own output alone; silu of
    large negative arguments is 0, not NaN."""
    for m, f32 in ((1, True), (2, False), (40, False)):
        p = Problem(dev, m, 130, 256, "tensor", f32)
        bias = torch.zeros(130, device=dev)
        bias[3], bias[5], bias[7] = float("inf"), float("-inf"), float("nan")
        bias[9] = -1e30
        e = p.sh.sherry_epilogue()
        e.bias, e.act = bias.data_ptr(), p.sh.SHERRY_ACT_SILU
        y = torch.empty((m, 130), device=dev)
        p.call(e, y)
        y = y.cpu()
        assert bool((y[:, 3] == float("inf")).all()) and bool(torch.isnan(y[:, 7]).all())
        assert bool(torch.isnan(y[:, 5]).all())  # -inf * 0, as the formula gives
        assert bool((y[:, 9] == 0).all())
        rest = [i for i in range(130) if i not in (3, 5, 7)]
        assert bool(torch.isfinite(y[:, rest]).all())


def test_captured_epilogue(dev):
    """In a graph on a stream of its own, replayed, against the eager result."""
    p = Problem(dev, 1, 514, 2052, "channel", True)
    p2 = Problem(dev, 40, 514, 644, "group", False)
    res = [torch.randn((m, 514), device=dev) for m in (1, 40)]
    es = []
    for r in res:
        e = p.sh.sherry_epilogue()
        e.residual, e.act = r.data_ptr(), p.sh.SHERRY_ACT_GELU
        es.append(e)
    y = [torch.zeros((m, 514), device=dev) for m in (1, 40)]
    p.call(es[0], y[0])
    p2.call(es[1], y[1])
    want = [t.clone() for t in y]
    sh = p.sh
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        sh.sherry_gemv_f32_epilogue(p.w, p.x, p.sx, *p.ws, es[0], y[0], p.n, p.k)
        sh.sherry_gemm_epilogue(p2.w, p2.x, p2.sx, *p2.ws, es[1], y[1], p2.m, p2.n, p2.k)
    for _ in range(3):
        for t in y:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(y, want))
        assert float(torch.randn(1000, device=dev).sum()) < 1e9


@pytest.mark.parametrize("m,f32", [(1, True), (3, False), (40, False)])
@pytest.mark.parametrize("act", ACTS)
def test_activations_relative_error(dev, m, f32, act):
    """act(z) of chosen z (a product of 0 and a bias) within the header's relative
    bounds, out to where its result is 2^-116: 1 ulp = 2u each of the exp2 and
    reciprocal units and u of each operation make 8u of silu; gelu adds its
    polynomial's 1.8u, its argument's 3u and Horner's 2u (16u).  Below 0 an exponent
    -E (in units of ln 2) whose factors and products are rounded c times adds
    c E ln 2 u: silu's 1.3 |z|, gelu's 2.3 z^2 / 2, gelu_tanh's 6 w."""
    import paper_2601_07892_amd as sh
    from scipy.special import erfc, expit
    n, k, low = 32768, 128, {"silu": -84, "gelu": -12.5, "gelu_tanh": -9}.get(act, -1e18)
    rng = np.random.default_rng(5)
    z = np.concatenate([rng.uniform(max(low, -100), 100, n // 4), rng.uniform(max(low, -13), -1, n // 4), rng.uniform(-2, 2, n // 4),
                        np.exp(rng.uniform(-20, np.log(-low), n // 8)) * -1, np.exp(rng.uniform(-20, 40, n // 8))]).astype(np.float32)
    w = torch.from_numpy(sh.sherry_pack(synth.ternary_34(n, k, 15, "zero"))).to(dev)
    x = torch.zeros((m, k), device=dev) if f32 else torch.zeros((m, k), dtype=torch.int8, device=dev)
    sx, bias, y = torch.ones(m, device=dev), torch.from_numpy(z).to(dev), torch.empty((m, n), device=dev)
    e = sh.sherry_epilogue()
    e.act, e.bias = getattr(sh, "SHERRY_ACT_" + act.upper()), bias.data_ptr()
    if f32:
        sh.sherry_gemv_f32_epilogue(w, x, sx, 1.0, None, None, e, y, n, k)
    else:
        sh.sherry_gemm_epilogue(w, x, sx, 1.0, None, None, e, y, m, n, k)
    torch.cuda.synchronize()
    z = z.astype(np.float64)
    arg = 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)
    want = {"gelu": lambda: 0.5 * z * erfc(-z / np.sqrt(2)), "gelu_tanh": lambda: z * expit(arg)}.get(act, lambda: _act(z, act))()
    under = np.minimum(z, 0)
    bound = {"none": 0, "relu": 0, "relu2": 1, "silu": 8 - 2 * under, "gelu": 16 + 2 * under ** 2,
             "gelu_tanh": 8 + 8 * np.maximum(0, -arg)}[act] * U
    assert np.abs(want[want != 0]).min() > 2.0 ** -116 or act in ("relu", "none")
    assert np.all(np.abs(y.double().cpu().numpy() - want) <= bound * np.abs(want))
