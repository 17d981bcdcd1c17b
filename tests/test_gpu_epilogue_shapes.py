"""GPU parity of the epilogue in every shape of the register-decoded kernel, apart
and in place, against 64 bits on the library's own product without one (which is
bit for bit what the epilogue starts from, and is tested elsewhere).

Tolerance (u = 2^-24), the product being exact here: u |z| for the bias, passed
on by the activation's slope; 8 u |z| of the activation; u each for the gate and
the residual."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from test_gpu_epilogue import ACTS, U, dev  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# (m, n, k): long, mid, half, quarter, short, tiny workgroups; rows that are and that
# are not whole 16-byte pieces
LONE = [(1025, 4100, 1028), (2049, 2051, 1028), (1025, 2052, 132), (700, 3077, 260), (2049, 514, 132),
        (2049, 516, 132), (1025, 1028, 4100), (513, 2050, 4100), (130, 1032, 256), (40, 1028, 4100)]
# with per-group scales mid, half, pair, short, tiny, whose scales are read one unit
# and (units a multiple of four) four units at a time
LONE_GROUP = [(1025, 2052, 132), (1025, 4100, 1028), (700, 3077, 500), (1025, 2052, 500), (513, 2052, 2052),
              (513, 2050, 2052), (1025, 1028, 1924), (130, 1030, 256), (130, 1028, 500), (16, 300, 2048), (40, 1028, 4100)]


def _act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "relu2":
        return z.clamp(min=0) ** 2
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z * 0.5 ** 0.5)
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3))
    return z


class Product:
    def __init__(self, dev, m, n, k, scales):
        import paper_2601_07892_amd as sh
        import synth
        self.sh, self.m, self.n, self.k, self.dev = sh, m, n, k, dev
        g = self.g = torch.Generator(device=dev)
        g.manual_seed(m * 31 + n * 7 + k)
        self.w = torch.from_numpy(sh.sherry_pack(synth.ternary_34(n, k, 15, "shapes"))).to(dev)
        self.x = torch.randint(-127, 128, (m, k), generator=g, device=dev, dtype=torch.int8)
        self.sx = torch.rand(m, generator=g, device=dev) * 0.01 + 0.001
        shape = {"channel": (n,), "group": (n, -(-k // 128))}[scales]
        s = torch.rand(shape, generator=g, device=dev) * (0.3 / k ** 0.5) + 1e-3
        self.ws = (0.0, s, None) if scales == "channel" else (0.0, None, s)

    def call(self, e, y):
        self.sh.sherry_gemm_epilogue(self.w, self.x, self.sx, *self.ws, e, y, self.m, self.n, self.k)
        torch.cuda.synchronize()

    def randn(self, *shape):
        return torch.randn(shape, generator=self.g, device=self.dev)

    def check(self, act, bias, gate, residual):
        sh, m, n = self.sh, self.m, self.n
        p = torch.empty((m, n), device=self.dev)
        self.call(sh.sherry_epilogue(), p)
        b, g, r = self.randn(n) if bias else None, self.randn(m, n) if gate else None, self.randn(m, n) if residual else None
        e = sh.sherry_epilogue()
        e.act = getattr(sh, "SHERRY_ACT_" + act.upper())
        e.bias, e.gate, e.residual = (None if t is None else t.data_ptr() for t in (b, g, r))
        flat = torch.full((m * n + 8,), float("nan"), device=self.dev)
        y = flat[:m * n].view(m, n)
        self.call(e, y)
        assert bool(torch.isnan(flat[m * n:]).all())
        z = p.double() + (b.double() if bias else 0)
        a = _act64(z, act)
        slope = 2 * z.abs() if act == "relu2" else 1.2
        own = 0 if act == "none" else 8 * U * (z * z if act == "relu2" else z.abs())
        err = slope * U * z.abs() * bool(bias) + own
        if gate:
            a = a * g
            err = err * g.abs() + U * a.abs()
        if residual:
            a = a + r
            err = err + U * a.abs()
        assert not bool(((y.double() - a).abs() > 1.01 * err + 1e-37).any())
        # in place: y is what the epilogue reads
        for name, t in (("gate", g), ("residual", r)):
            if t is not None:
                own_y = t.clone()
                setattr(e, name, own_y.data_ptr())
                self.call(e, own_y)
                assert torch.equal(own_y, y), name
                setattr(e, name, t.data_ptr())


@pytest.mark.parametrize("scales,m,n,k", [("channel",) + s for s in LONE] + [("group",) + s for s in LONE_GROUP])
def test_epilogue_of_every_shape(dev, scales, m, n, k):
    print("[case] epilogue shapes", scales, m, n, k, file=sys.stderr, flush=True)
    p = Product(dev, m, n, k, scales)
    for i, (bias, gate, residual) in enumerate([(1, 1, 0), (0, 1, 1), (1, 0, 1)]):
        p.check(ACTS[(i + m + n) % 6], bias, gate, residual)
