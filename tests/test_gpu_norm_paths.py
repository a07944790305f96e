"""Group norm's paths at sizes that reach all of each, against the definition
in 64 bits on the GPU: thread blocks that take several slabs, where one ends
inside a block, on every vector width; rows in blocks; column passes.
Tolerances as in test_gpu_norm.py, h's error that of a subtraction first (4 U |h|)."""

import pytest

from .gpu_common import lib_ready, torch_cuda
from .test_gpu_norm import U

pytestmark = pytest.mark.gpu

SHAPES = [
    (512, 196, 64, 4), (333, 196, 128, 8), (601, 49, 120, 8), (500, 64, 512, 32), (900, 49, 256, 32), (700, 100, 96, 3),
    (300, 784, 64, 8), (1000, 33, 70, 7), (257, 90, 198, 3),  # slabs
    (1500, 1, 8192, 2), (1300, 1, 1120, 32), (900, 3, 500, 10),  # rows
    (40, 1000, 130, 2), (5, 20001, 24, 3),  # columns
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_definition(shape, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    k = SHAPES.index(shape)
    kind = ("silu", "none", "relu")[k % 3]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    gen = torch.Generator(device="cuda").manual_seed(k)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x = (2 * rand(n, S, C) + rand(C)).to(dt)
    gamma, beta = 1 + 0.3 * rand(C), 0.3 * rand(C)
    dy = (rand(n, S, C) + 0.5).to(dt)

    def groups(t):
        return t.view(n, S, G, C // G)

    def avg(t):
        return groups(t).mean((1, 3))[:, None, :, None].expand(n, S, G, C // G).reshape(n, S, C)

    def wide(t):
        return t.double()[:, None, :, None].expand(n, S, G, C // G).reshape(n, S, C)

    x64, g64, b64 = x.double(), gamma.double(), beta.double()
    y, m, r = ff.group_norm_act(x, gamma, beta, G, act=kind, eps=1e-5)
    mean = groups(x64).mean((1, 3))
    rstd = (groups(x64).var((1, 3), unbiased=False) + 1e-5) ** -0.5
    ax = groups(x64).abs().mean((1, 3))
    assert bool(((m.double() - mean).abs() <= 64 * U * ax + 1e-30).all())
    assert bool(((r.double() - rstd).abs() <= 64 * U * rstd * (1 + (ax * rstd) ** 2 * U * 64)).all())

    def sig(u):
        return torch.sigmoid(u)

    u = (x64 - wide(mean)) * wide(rstd) * g64 + b64
    DU = 80 * U * (g64.abs() * wide(rstd) * (x64.abs() + wide(ax)) + b64.abs())
    y64 = u * sig(u) if kind == "silu" else u.clamp(min=0) if kind == "relu" else u
    assert bool(((y.double() - y64).abs() <= 1.1 * DU + (half + 2.0 ** -20) * y64.abs() + 1e-30).all())

    # the gradient, with the forward's own mean and rstd as its inputs
    R = wide(r)
    h = (x64 - wide(m)) * R
    u = h * g64 + b64
    DH = 4 * U * h.abs()
    DUU = g64.abs() * DH + 4 * U * (u.abs() + b64.abs())
    dy[u.abs() <= DUU] = 0  # no gradient at the ReLU's kink, where either side is right
    d64 = dy.double()
    dx, dgam, dbet = ff.group_norm_act_backward(dy, x, m, r, gamma, beta, G, act=kind)
    slope = sig(u) * (1 + u * (1 - sig(u))) if kind == "silu" else (u > 0).double() if kind == "relu" else 1.0
    du = d64 * slope
    # bf16: the exponential's argument, below 20 here, is rounded to 2^-24 of itself; p (1 + |u|) bounds what cancels
    rel = 4 * U + (2.0 ** -17 if dtype == "bf16" else 2.0 ** -20)
    Ddu = d64.abs() * (0.5 * DUU + rel * (1.1 + sig(u) * u.abs())) if kind == "silu" else 0 * d64
    tb = Ddu.sum((0, 1)) + 64 * U * du.abs().sum((0, 1))
    tg = (Ddu * h.abs() + du.abs() * DH).sum((0, 1)) + 64 * U * (du * h).abs().sum((0, 1))
    assert bool(((dbet.double() - du.sum((0, 1))).abs() <= tb + 1e-30).all())
    assert bool(((dgam.double() - (du * h).sum((0, 1))).abs() <= tg + 1e-30).all())
    w, Dw = g64 * du, g64.abs() * Ddu
    a1, a2 = avg(w), avg(w * h)
    D1 = avg(Dw) + 64 * U * avg(w.abs())
    D2 = avg(Dw * h.abs() + w.abs() * DH) + 64 * U * avg((w * h).abs())
    dx64 = R * (w - a1 - h * a2)
    tol = R * (Dw + D1 + h.abs() * D2 + DH * a2.abs() + 4 * U * (w.abs() + a1.abs() + (h * a2).abs()))
    assert bool(((dx.double() - dx64).abs() <= tol + half * dx64.abs() + 1e-30).all())
